"""GELU of float results far below zero, on the GPU: small results are right to a share of themselves, not of z."""
import numpy as np
import pytest

import block_util as bu
from oracle import block

pytestmark = pytest.mark.gpu
# normal_tail_far's error in float arithmetic, with as much again for the last bits of the exponential (2^-22 of an argument of up to 126 is 3e-5 there)
TAIL = 2.1e-5 + 3e-5


def layer(M, K, values):
    """Y = act(X I): Z is X to the bit, whichever tile computes it."""
    rng = np.random.default_rng(M)
    job = bu.dense_job(rng, M, K, K, act=block.GELU, out="f32", bias=False, residual=False)
    z = bu.bf16(np.resize(values, M * K)).reshape(M, K)
    job["parts"][2].update(x=z, w=np.eye(K))
    rnd = bu.run_dense([job])
    y = rnd.read(0, "y")
    rnd.close()
    return z, y


@pytest.mark.parametrize("M,K", [(1, 1024), (20, 72), (200, 264), (300, 1024), (3000, 1032)])
def test_negative_tail(M, K):
    z, y = layer(M, K, -np.linspace(0.0, 12.88, 4999))
    want = block.act(z, block.GELU)
    off = np.abs(y - want) / np.maximum(np.abs(want), 1e-37)
    assert (off <= TAIL).all(), (off.max(), z.flat[off.argmax()])


def test_ends():
    """Nothing is left of a very negative number or of minus infinity (the limit), large ones and infinity pass, a NaN stays one."""
    values = np.array([-1e30, -100.0, -14.0, -np.inf, np.nan, 0.0, 14.0, 1e30, np.inf])
    # rows of one number each beside zeros: infinity times the other weights' zeros is a NaN, so the diagonal is all there is
    rng = np.random.default_rng(2)
    job = bu.dense_job(rng, len(values), 8, 8, act=block.GELU, out="f32", bias=False, residual=False)
    x = np.zeros((len(values), 8))
    x[:, 3] = values
    job["parts"][2].update(x=x, w=np.ones((8, 8)))
    rnd = bu.run_dense([job])
    y = rnd.read(0, "y")[:, 5]
    rnd.close()
    assert (np.abs(y[:4]) <= 1e-37).all() and np.isnan(y[4]) and y[5] == 0 and y[8] == np.inf
    assert np.abs(y[6:8] / bu.bf16(values[6:8]) - 1).max() <= 4 * block.STEP
