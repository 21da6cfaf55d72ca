"""What the calls on 8-bit integers refuse, without a GPU: every check comes before anything is enqueued."""
import ctypes as C

import pytest
import torch

from paper_2605_17633_amd import binding as B

P = C.c_void_p(4096)          # never followed: a call that is refused touches no buffer
ODD = C.c_void_p(4104)
NULL = C.c_void_p(0)


def linear(A=P, lda=64, a_scales=P, W=P, ldw=64, w_scales=P, bias=P, Cm=P, ldc=32, M=4, N=32, K=64, epi=B.EPI_BIAS_SCATTER_ADD, row_map=P, rows=4, stride=4, dst=8):
    return B.lib().ssam_linear_i8(A, lda, a_scales, W, ldw, w_scales, bias, Cm, ldc, M, N, K, epi, row_map, rows, stride, dst, None)


@pytest.mark.parametrize("bad", [{name: p} for name in ("A", "a_scales", "W", "w_scales", "bias", "Cm") for p in (NULL, ODD)] +
                         [dict(M=0), dict(N=0), dict(K=-1), dict(lda=48), dict(ldw=48), dict(ldc=24), dict(lda=72), dict(ldw=72), dict(ldc=36), dict(epi=-1), dict(epi=4),
                          dict(row_map=NULL), dict(rows=0), dict(stride=-1), dict(dst=0)])
def test_linear_refuses(bad):
    assert linear(**bad) == B.EINVAL


@pytest.mark.parametrize("bad", [dict(N=28), dict(K=56), dict(K=131072, lda=131072, ldw=131072), dict(lda=(1 << 22) + 16), dict(ldw=(1 << 22) + 16),
                                 dict(M=2 ** 31 - 65536, N=128, ldc=128),
                                 dict(M=2 ** 31 - 65535), dict(M=1, N=2 ** 31 - 65528, ldc=2 ** 31 - 65528), dict(M=1 << 20, rows=1, stride=1, dst=1 << 11)])
def test_linear_refuses_sizes(bad):
    assert linear(**bad) == B.EUNSUPPORTED


@pytest.mark.parametrize("rows,D,want", [(0, 64, B.EINVAL), (-1, 64, B.EINVAL), (4, 0, B.EINVAL), (4, 56, B.EUNSUPPORTED), (1, 131072, B.EUNSUPPORTED), (1 << 40, 16, B.EUNSUPPORTED)])
def test_quantize_refuses_sizes(rows, D, want):
    assert B.lib().ssam_quantize_rows(P, P, P, C.c_long(rows), C.c_int(D), None) == want


@pytest.mark.parametrize("k", range(3))
@pytest.mark.parametrize("bad", [NULL, ODD])
def test_quantize_refuses_pointers(bad, k):
    args = [P] * 3
    args[k] = bad
    assert B.lib().ssam_quantize_rows(*args, C.c_long(4), C.c_int(64), None) == B.EINVAL


def test_binding_refuses():
    x, c, f = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    for call in (lambda: B.ssam_quantize_rows(x), lambda: B.ssam_linear_i8(c, f, c, f, f)):
        with pytest.raises(TypeError):
            call()                               # tensors of the host
    for call in (lambda: B.ssam_linear_i8(c, f, c[:, :32], f, f), lambda: B.ssam_linear_i8(c, f[:1], c, f, f), lambda: B.ssam_linear_i8(c, f, c, f, f[:1]),
                 lambda: B.ssam_linear_i8(c, f, c, f, f, epilogue=B.EPI_BIAS_SCATTER)):
        with pytest.raises(ValueError):
            call()
