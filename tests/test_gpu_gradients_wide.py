"""Gradient of the LayerNorm of wide rows, so many that every wave takes several: each number of chunks a lane, added and written, against 64 bits."""
import pytest
import torch

import test_gpu_gradients as T
from helpers import announce
from paper_2605_17633_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("Bn,N,Nout,D", [(2, 4000, 4100, 2048), (1, 9000, 8900, 1544), (3, 2000, 2100, 1536), (2, 3500, 3333, 1032), (1, 12000, 12000, 520)])
def test_several_rows_a_wave(Bn, N, Nout, D, accumulate):
    """512 workgroups of four waves: up to 6 rows a wave, whose sums are followed by four waves' and 512 workgroups' in 32 shares: under 64 additions in a row of 2^-24, and the error of h."""
    announce("ln_gather_backward several rows a wave", Bn, N, Nout, D, accumulate)
    x, idx, gamma, dy, dx0 = T.ln_inputs(Bn, N, Nout, D, True, D)
    dx, dgamma, dbeta = B.ssam_ln_gather_backward(x, idx, Nout, gamma, T.EPS, dy, dx=dx0.clone(), accumulate=accumulate)
    ref, rg, rb, slack, mg, mb = T.ln_reference(x, idx, gamma, dy, dx0, accumulate)
    T.close(dx, ref, slack, "dx")
    untouched = slack.amax(2) == 0
    assert torch.equal(dx[untouched], dx0[untouched])
    for got, want, size in ((dgamma, rg, mg), (dbeta, rb, mb)):
        assert ((got.double() - want).abs() <= 2.0 ** -18 * size + 1e-30).all()
    again = B.ssam_ln_gather_backward(x, idx, Nout, gamma, T.EPS, dy, dx=dx0.clone(), accumulate=accumulate)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))
