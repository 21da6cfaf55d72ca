"""Activations in 8 bits: the codes themselves, ties to even among them, against whole-number arithmetic."""
import pytest
import torch

from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, BF = "cuda", torch.bfloat16


def whole(x):
    """bf16 [rows, D] -> mantissas and exponents: x = m * 2^e, m a whole number below 2^8"""
    bits = x.view(torch.int16).long() & 0xffff
    exp, frac = (bits >> 7) & 0xff, bits & 0x7f
    m = torch.where(exp > 0, frac + 128, frac)
    return torch.where(bits >= 0x8000, -m, m), exp.clamp(min=1) - 134


def codes_of(x):
    """rint(127 x / top), ties to even, of every 64 columns: quotients of whole numbers"""
    rows, D = x.shape
    m, e = whole(torch.nn.functional.pad(x, (0, -D % 64)))
    m, e = m.view(rows, -1, 64), e.view(rows, -1, 64)
    at = torch.where(m != 0, m.abs() + (e << 8), -(1 << 20)).argmax(2, keepdim=True)             # (mantissas below 2^7 have the least exponent)
    mt, et = m.gather(2, at).abs(), e.gather(2, at)
    down = (et - e).clamp(0, 20)                          # beyond that a code is 0 in any case
    num, den = 2 * 127 * m.abs(), (mt << down).clamp(min=1)
    twice = num // den                                    # floor of twice the quotient: odd and exact is a tie
    code = (twice + 1) // 2
    tie = (twice % 2 == 1) & (num % den == 0)
    code = torch.where(tie & (code % 2 == 1), code - 1, code)
    return (code * m.sign()).view(rows, -1)[:, :D].to(torch.int8)


@pytest.mark.parametrize("rows,D", [(1, 8), (7, 144), (300, 1000), (2048, 5120)])
def test_codes(rows, D):
    announce("checkpoint codes", rows, D)
    g = torch.Generator(device=DEV)
    g.manual_seed(D)
    x = (torch.randn(rows, D, generator=g, device=DEV) * torch.exp(2 * torch.randn(rows, 1, generator=g, device=DEV))).to(BF)
    got = B.ssam_checkpoint_store(x)[0]
    assert torch.equal(got, codes_of(x))
    assert torch.equal(B.ssam_gelu_checkpoint(x)[1], got)


def test_ties():
    """Every bf16 value below every largest one of two binades: with a mantissa of 254 every half is one of them."""
    announce("checkpoint ties")
    top = torch.arange(0x3f80, 0x4080, dtype=torch.int32, device=DEV)
    values = torch.arange(0x3a80, 0x4080, dtype=torch.int32, device=DEV)
    x = values.repeat(256, 1)
    x = torch.where(x > top[:, None], top[:, None], x)
    blocks = torch.cat([top[:, None, None].expand(-1, x.shape[1] // 32, 1), x.view(256, -1, 32), (x | 0x8000).view(256, -1, 32)[:, :, 1:]], 2).reshape(256, -1)
    x = torch.where(blocks >= 0x8000, blocks - 0x10000, blocks).to(torch.int16).view(BF).contiguous()
    assert x.shape[1] % 64 == 0
    got, want = B.ssam_checkpoint_store(x)[0], codes_of(x)
    halves = (x.double().abs() * 254 / (x.double().abs().view(256, -1, 64).amax(2, keepdim=True).expand(-1, -1, 64).reshape(256, -1))) % 2 == 1
    assert int(halves.sum()) > 100
    assert torch.equal(got, want)
