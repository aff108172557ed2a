"""The gate's slope where it is small, on the GPU: every kind of tile within 8 steps of 2^-24 (1 + |z|) of it, as a dense layer's (before the rounding of [dG dU])."""
import numpy as np
import pytest

import block_util as bu
from oracle import block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [block.GELU, block.SILU])
@pytest.mark.parametrize("M,K,F,N", [(4, 64, 136, 8), (40, 72, 264, 8), (128, 8, 264, 264), (128, 8, 1032, 8), (500, 8, 264, 8), (2048, 8, 4096, 8)])
def test_slopes(M, K, F, N, act):
    """One row of the weights carries dX and dW_in, so that no sum hides what a factor is off by."""
    rng = np.random.default_rng(M + act)
    job = bu.gated_job(rng, M, K, F, N, act=act, train=True, residual=False, scale=1.0)
    d = job["parts"][2]
    x = np.zeros((M, K))
    x[np.arange(M), np.arange(M) % K] = bu.bf16(rng.uniform(-9, 9, M))      # the gate is x times a weight
    w_in = np.zeros((K, 2 * F))
    w_in[:, :F] = bu.bf16(rng.uniform(0.2, 1.0, (K, F)))
    w_in[:, F:] = bu.bf16(rng.standard_normal((K, F)))
    d.update(x=x, w_in=w_in)
    rnd = bu.run_gated([job])
    h, gu = rnd.read(0, "h"), rnd.read(0, "gu")
    want = block.gated_backward(x, w_in, d["w_out"], h, gu, d["dy"], act, fine=True)
    bu.within(rnd.read(0, "dx"), want["dx"], "dx", 0)
    bu.within(rnd.read(0, "dw_in"), want["dw_in"], "dw_in", 0)
    rnd.close()
