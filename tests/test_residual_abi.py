"""What the step between two halves of a block, its gradient and the inverse tables refuse, without a GPU: every check comes before anything is enqueued."""
import ctypes as C

import pytest
import torch

from paper_2605_17633_amd import binding as B

P = C.c_void_p(4096)          # never followed: a call that is refused touches no buffer
Q = C.c_void_p(8192)
ODD = C.c_void_p(4104)
NULL = C.c_void_p(0)


def forward(x=P, x_out=Q, o=P, src=P, src_stride=0, post_g=P, post_b=P, gate=P, gate_stride=0, pre_g=P, pre_b=P, dst=P, dst_stride=0, eps=1e-6, y=P, scales=P,
            Bn=2, N=10, No=8, Ny=6, D=64, eight=False):
    head = (x, x_out, o, src, src_stride, post_g, post_b, gate, gate_stride, C.c_float(1), pre_g, pre_b, dst, dst_stride, C.c_float(eps), y)
    if eight:
        return B.lib().ssam_residual_norm_i8(*head, scales, Bn, N, No, Ny, D, None)
    return B.lib().ssam_residual_norm(*head, Bn, N, No, Ny, D, None)


def backward(x=P, o=P, src=P, src_stride=0, post_g=P, post_b=P, gate=P, gate_stride=0, pre_g=P, dst=P, dst_stride=0, eps=1e-6, dy=P, dx_out=P, dx=Q, do=P,
             dgate=P, dpost_g=P, dpost_b=P, dpre_g=P, dpre_b=P, Bn=2, N=10, No=8, Ny=6, D=64, ws=P, ws_bytes=1 << 40):
    return B.lib().ssam_residual_norm_backward(x, o, src, src_stride, post_g, post_b, gate, gate_stride, C.c_float(1), pre_g, dst, dst_stride, C.c_float(eps), dy, dx_out, dx, do,
                                               dgate, dpost_g, dpost_b, dpre_g, dpre_b, Bn, N, No, Ny, D, ws, C.c_size_t(ws_bytes), None)


SIZES = [dict(Bn=0), dict(N=0), dict(No=0), dict(Ny=-1), dict(D=0), dict(D=60), dict(src_stride=9), dict(src_stride=-1), dict(dst_stride=9), dict(gate_stride=63), dict(gate_stride=66),
         dict(src=NULL), dict(dst=NULL), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan"))]


@pytest.mark.parametrize("bad", SIZES + [dict(x=NULL), dict(x_out=NULL), dict(post_b=NULL), dict(post_g=NULL), dict(pre_b=NULL), dict(pre_g=NULL), dict(y=NULL), dict(o=NULL),
                                         dict(x=ODD), dict(x_out=ODD), dict(o=ODD), dict(post_g=ODD), dict(post_b=ODD), dict(gate=ODD), dict(pre_g=ODD), dict(pre_b=ODD), dict(y=ODD)])
@pytest.mark.parametrize("eight", [False, True])
def test_forward_refuses(bad, eight):
    assert forward(**bad, eight=eight) == B.EINVAL


def test_forward_refuses_combinations():
    nothing = dict(o=NULL, src=NULL, post_g=NULL, post_b=NULL, gate=NULL)
    assert forward(**nothing, pre_g=NULL, pre_b=NULL, dst=NULL, y=NULL) == B.EINVAL             # neither a branch nor a norm
    assert forward(**nothing) == B.EINVAL                                                       # without a branch the stream is not copied
    assert forward(**nothing, x_out=P, gate_stride=0, D=2056) == B.EUNSUPPORTED                  # (x itself may be given)
    assert forward(D=2056) == B.EUNSUPPORTED and forward(Bn=1 << 16, N=1 << 15) == B.EUNSUPPORTED
    assert forward(D=72, eight=True) == B.EUNSUPPORTED and forward(scales=NULL, eight=True) == B.EINVAL and forward(scales=ODD, eight=True) == B.EINVAL
    assert forward(pre_g=NULL, pre_b=NULL, dst=NULL, y=NULL, eight=True) == B.EINVAL


@pytest.mark.parametrize("bad", SIZES + [dict(x=NULL), dict(dx=NULL), dict(do=NULL), dict(o=NULL), dict(dy=NULL), dict(pre_g=NULL), dict(post_g=NULL), dict(post_b=NULL), dict(gate=NULL),
                                         dict(x=ODD), dict(o=ODD), dict(dy=ODD), dict(dx_out=ODD), dict(dx=ODD), dict(do=ODD), dict(dgate=ODD), dict(dpost_g=ODD), dict(dpre_b=ODD),
                                         dict(ws=NULL), dict(ws=ODD)])
def test_backward_refuses(bad):
    assert backward(**bad) == B.EINVAL


def test_backward_refuses_sizes():
    need = B.ssam_residual_norm_backward_workspace_bytes
    assert backward(D=2056) == B.EUNSUPPORTED and backward(Bn=1 << 16, N=1 << 15) == B.EUNSUPPORTED
    assert need(2, 10, 64) > 0 and backward(ws_bytes=need(2, 10, 64) - 1) == B.EWORKSPACE
    assert backward(gate_stride=64, ws_bytes=need(2, 10, 64, 2) - 1) == B.EWORKSPACE
    assert need(0, 10, 64) == need(2, 10, 64, 3) == need(2, 0, 64) == 0
    assert backward(Bn=65536, N=1, No=1, Ny=1, gate_stride=64) == B.EUNSUPPORTED


@pytest.mark.parametrize("bad,want", [(dict(idx=NULL), B.EINVAL), (dict(inv=NULL), B.EINVAL), (dict(Bn=0), B.EINVAL), (dict(Nout=0), B.EINVAL), (dict(N=-1), B.EINVAL),
                                      (dict(stride=7), B.EINVAL), (dict(Bn=1 << 16, N=1 << 15), B.EUNSUPPORTED), (dict(Bn=1 << 16, Nout=1 << 15), B.EUNSUPPORTED)])
def test_invert_rows_refuses(bad, want):
    a = dict(idx=P, stride=0, inv=Q, Bn=2, Nout=8, N=10) | bad
    assert B.lib().ssam_invert_rows(*a.values(), None) == want


def test_binding_refuses():
    x = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    for call in (lambda: B.ssam_residual_norm(x, pre=(torch.ones(64), torch.ones(64))), lambda: B.ssam_residual_norm_i8(x), lambda: B.ssam_residual_norm_backward(x),
                 lambda: B.ssam_invert_rows(torch.zeros(3, dtype=torch.int32), 4)):
        with pytest.raises(TypeError):
            call()                               # tensors of the host
