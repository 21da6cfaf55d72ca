"""Sizes that no C int holds are refused by the binding of the 8-bit calls and of the step: ctypes would cut them to 32 bits and the call would do a part of its work.
Without a GPU: tensors without memory, and a library that records what reaches it."""
import pytest
import torch

from paper_2605_17633_amd import binding as B

MORE = 2 ** 32                # cut to 32 bits: nothing of it is left


@pytest.fixture
def reached(monkeypatch):
    real, calls = B.lib(), []

    class Recorder:
        ssam_status_string = real.ssam_status_string

        def __getattr__(self, name):
            def call(*args):
                calls.append((name, args))
                return 0
            return call

    recorder = Recorder()
    monkeypatch.setattr(B, "lib", lambda: recorder)
    monkeypatch.setattr(B, "_here", lambda t, name: -1)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)
    return calls


def meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def i8(*shape):
    return meta(*shape, dtype=torch.int8)


def f32(*shape):
    return meta(*shape, dtype=torch.float32)


def i32(*shape):
    return meta(*shape, dtype=torch.int32)


def refused(call, reached):
    with pytest.raises(B.SsamError) as e:
        call()
    assert e.value.code == B.EUNSUPPORTED and not reached


def linear(M=32, N=64, K=64, A=None, W=None, C=None, **k):
    return B.ssam_linear_i8(i8(M, K) if A is None else A, f32(M), i8(N, K) if W is None else W, f32(N), f32(N), C, **k)


def scatter(rows=32, stride=32, dst=32, M=32):
    row_map = i32(max(stride, rows) * max(1, -(-M // rows)))
    return linear(M=M, C=meta(max(dst, 32) * max(1, -(-M // rows)), 64), epilogue=B.EPI_BIAS_SCATTER, row_map=row_map, rows_per_batch=rows, map_batch_stride=stride, dst_rows_per_batch=dst)


@pytest.mark.parametrize("call", [
    lambda: B.ssam_quantize_rows(meta(1, MORE + 64)), lambda: B.ssam_quantize_rows(meta(2 ** 31)),
    lambda: linear(M=MORE + 32), lambda: linear(N=MORE + 64), lambda: linear(K=MORE + 64), lambda: linear(M=2 ** 31),
    lambda: linear(A=i8(32, MORE + 64)[:, :64]), lambda: linear(W=i8(64, MORE + 64)[:, 64:128]), lambda: linear(C=meta(32, MORE + 64)[:, :64]),
    lambda: scatter(rows=MORE + 32), lambda: scatter(stride=MORE + 32), lambda: scatter(dst=MORE + 32),
    lambda: B.ssam_invert_rows(i32(8), MORE + 8), lambda: B.ssam_invert_rows(i32(MORE + 8), 8), lambda: B.ssam_invert_rows(i32(MORE + 1, 8), 8),
])
def test_8_bits_and_tables(call, reached):
    refused(call, reached)


PRE = (f32(64), f32(64))


@pytest.mark.parametrize("step", [B.ssam_residual_norm, B.ssam_residual_norm_i8])
@pytest.mark.parametrize("k", [dict(x=meta(1, MORE + 8, 64)), dict(x=meta(MORE + 1, 8, 64)), dict(x=meta(1, 8, MORE + 64), pre=(f32(MORE + 64), f32(MORE + 64))),
                               dict(x=meta(1, 8, 64), o=meta(1, MORE + 8, 64), src=i32(8)), dict(x=meta(1, 8, 64), dst=i32(8), Ny=MORE + 8), dict(x=meta(1, 2 ** 31, 64))])
def test_step(step, k, reached):
    refused(lambda: step(**{"pre": PRE, **k}), reached)


@pytest.mark.parametrize("k", [dict(x_out=meta(1, MORE + 8, 64), dy=meta(1, MORE + 8, 64)), dict(x_out=meta(1, 8, 64), dy=meta(1, MORE + 8, 64), dst=i32(8)),
                               dict(x_out=meta(1, 8, 64), dy=meta(1, 8, 64), o=meta(1, MORE + 8, 64), src=i32(8))])
def test_gradients(k, reached):
    refused(lambda: B.ssam_residual_norm_backward(pre=PRE, **k), reached)


def test_workspace():
    need = B.ssam_residual_norm_backward_workspace_bytes
    assert need(1, MORE + 8, 64) == need(MORE + 1, 8, 64) == need(1, 8, MORE + 64) == need(MORE + 1, 8, 64, MORE + 1) == 0 < need(1, 8, 64)


def test_sizes_that_fit_reach_the_library(reached):
    B.ssam_quantize_rows(meta(MORE + 8, 64))              # (rows are a long)
    linear()
    scatter()
    B.ssam_invert_rows(i32(2, 8), 16)
    B.ssam_residual_norm(meta(1, 8, 64), meta(1, 8, 64), pre=PRE)
    B.ssam_residual_norm_i8(meta(1, 8, 64), meta(1, 8, 64), pre=PRE)
    B.ssam_residual_norm_backward(meta(1, 8, 64), meta(1, 8, 64), pre=PRE, dy=meta(1, 8, 64), weight_grads=False)
    assert [name for name, _ in reached] == ["ssam_quantize_rows", "ssam_linear_i8", "ssam_linear_i8", "ssam_invert_rows", "ssam_residual_norm", "ssam_residual_norm_i8", "ssam_residual_norm_backward"]
    assert reached[0][1][3] == MORE + 8
