"""Mapped epilogues of the 8-bit contraction on results that are column slices of a wider tensor, against 64 bits."""
import pytest
import torch

import residual_reference as R
from helpers import announce
from paper_2605_17633_amd import binding as B
from test_gpu_linear_i8 import BF, DEV, _check, _problem, _reference

pytestmark = pytest.mark.gpu


# few rows, of which 16 and 32 a workgroup, small and large tiles, and tiles of which the last are cut
@pytest.mark.parametrize("M,N,K", [(1, 72, 80), (20, 264, 208), (70, 520, 1040), (322, 232, 432), (700, 1288, 1040), (2105, 3880, 704), (3507, 4656, 480)])
@pytest.mark.parametrize("epi", [B.EPI_BIAS_SCATTER, B.EPI_BIAS_SCATTER_ADD])
def test_mapped(M, N, K, epi):
    """Rows of two images; what lies beside the slice, and rows that the map does not name, stay as they were."""
    announce("linear_i8 mapped slice", M, N, K, epi, B.lib().ssam_linear_i8_form(M, N, K, epi))
    A, sa, W, sw, bias = _problem(M, N, K, 12)
    gen = torch.Generator().manual_seed(M + epi)
    per = -(-M // 2)
    tokens, images = per + 2, -(-M // per)
    rows = torch.stack([torch.randperm(tokens, generator=gen)[:per] for _ in range(images)]).to(torch.int32)
    if per > 3:
        rows[:, 1], rows[:, 3] = -1, tokens
    old = torch.randn(images * tokens + 3, N + 24, generator=gen).to(BF)
    wide = old.to(DEV)
    B.ssam_linear_i8(A.to(DEV), sa.to(DEV), W.to(DEV), sw.to(DEV), bias.to(DEV), wide[1:images * tokens + 1, 8:8 + N], epilogue=epi, row_map=rows.to(DEV), rows_per_batch=per,
                     map_batch_stride=per, dst_rows_per_batch=tokens)
    got = wide.cpu()
    v, err = _reference(A, sa, W, sw, bias)
    m = rows.view(-1)[:M].long()
    there = (m >= 0) & (m < tokens)
    to = 1 + (torch.arange(M) // per * tokens + m)[there]
    ref = v[there] + (old[to, 8:8 + N].double() if epi == B.EPI_BIAS_SCATTER_ADD else 0)
    _check(got[to, 8:8 + N], ref, err[there] + R.U * ref.abs(), "mapped")
    got[to, 8:8 + N] = old[to, 8:8 + N]
    assert torch.equal(got, old)
