"""What the gradient calls refuse, without a GPU: every check comes before anything is enqueued."""
import ctypes as C

import pytest
import torch

from paper_2605_17633_amd import binding as B

P = C.c_void_p(4096)          # never followed: a call that is refused touches no buffer
ODD = C.c_void_p(4104)
NULL = C.c_void_p(0)


def ln(x=P, idx=P, stride=0, gamma=P, dy=P, dx=P, dgamma=P, dbeta=P, Bn=2, Nin=10, Nout=8, D=64, ws=P, ws_bytes=1 << 40):
    return B.lib().ssam_ln_gather_backward(x, idx, stride, gamma, C.c_float(1e-6), dy, dx, 1, dgamma, dbeta, Bn, Nin, Nout, D, ws, C.c_size_t(ws_bytes), None)


@pytest.mark.parametrize("bad", [dict(x=NULL), dict(idx=NULL), dict(gamma=NULL), dict(dy=NULL), dict(dx=NULL), dict(dgamma=NULL), dict(dbeta=NULL), dict(ws=NULL),
                                 dict(x=ODD), dict(gamma=ODD), dict(dy=ODD), dict(dx=ODD), dict(dgamma=ODD), dict(ws=ODD), dict(stride=7), dict(stride=-1),
                                 dict(Bn=0), dict(Nin=0), dict(Nout=-1), dict(D=0), dict(D=60)])
def test_layernorm_refuses(bad):
    assert ln(**bad) == B.EINVAL


def test_layernorm_refuses_sizes():
    assert ln(D=2056) == B.EUNSUPPORTED
    assert ln(Bn=1 << 16, Nout=1 << 15) == B.EUNSUPPORTED
    need = B.ssam_ln_gather_backward_workspace_bytes(2, 8, 64)
    assert need > 0 and ln(ws_bytes=need - 1) == B.EWORKSPACE
    assert B.ssam_ln_gather_backward_workspace_bytes(0, 8, 64) == 0


@pytest.mark.parametrize("rows,D,want", [(0, 64, B.EINVAL), (-1, 64, B.EINVAL), (4, 0, B.EINVAL), (4, 63, B.EINVAL), (1, (1 << 24) + 8, B.EUNSUPPORTED)])
def test_8_bit_calls_refuse_sizes(rows, D, want):
    L, n, D = B.lib(), C.c_long(rows), C.c_int(D)
    assert L.ssam_checkpoint_store(P, P, P, n, D, None) == want
    assert L.ssam_checkpoint_restore(P, P, P, n, D, None) == want
    assert L.ssam_gelu_checkpoint(P, P, P, P, n, D, None) == want
    assert L.ssam_gelu_backward(P, P, P, P, P, n, D, None) == want


@pytest.mark.parametrize("bad", [NULL, ODD])
def test_8_bit_calls_refuse_pointers(bad):
    L, n, D = B.lib(), C.c_long(4), C.c_int(64)
    for name, pointers in (("ssam_checkpoint_store", 3), ("ssam_checkpoint_restore", 3), ("ssam_gelu_checkpoint", 4), ("ssam_gelu_backward", 4)):
        for k in range(pointers):
            args = [P] * pointers
            args[k] = bad
            if name == "ssam_gelu_backward":
                args.append(P)                       # the activation, which may be NULL
            assert getattr(L, name)(*args, n, D, None) == B.EINVAL, (name, k)
    assert L.ssam_gelu_backward(P, P, P, P, ODD, n, D, None) == B.EINVAL


def test_binding_refuses_tensors_of_the_host():
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    for call in (lambda: B.ssam_checkpoint_store(x), lambda: B.ssam_gelu_checkpoint(x), lambda: B.ssam_checkpoint_restore(x, x),
                 lambda: B.ssam_gelu_backward(x, x, x),
                 lambda: B.ssam_ln_gather_backward(x[None], torch.zeros(2, dtype=torch.int32), 0, torch.ones(64), 1e-6, x[None])):
        with pytest.raises(TypeError):
            call()
