"""A NaN that the forward pass left in Z or in the gate, on the GPU: every gradient that it is a factor of is one, and no other.  dY is finite: nothing else
carries it."""
import numpy as np
import pytest

import block_util as bu
from oracle import block
from paper_1902_04610_amd import salus

pytestmark = pytest.mark.gpu
ACTS = [block.RELU, block.GELU, block.SILU]


def only(got, where):
    """NaN there and nowhere else."""
    want = np.zeros(got.shape, bool)
    want[where] = True
    assert np.array_equal(np.isnan(got), want), np.argwhere(np.isnan(got) != want)[:8].tolist()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", [(1, 8, 8), (5, 72, 40), (70, 136, 520), (300, 264, 264)])
def test_dense(M, K, N, act):
    rng = np.random.default_rng(M)
    jobs = [bu.dense_job(rng, M, K, N, act=act, train=True)]
    rnd = bu.run_dense(jobs)
    row, column = M // 2, N - 3
    z = rnd.read(0, "z")
    z[row, column] = np.nan
    rnd.load(0, "z", z)
    grads, keep = bu.dense_grad_descs(rnd, jobs)
    assert rnd.dp.pool.grouped_dense_backward(grads, stream=rnd.dp.stream) == salus.OK
    rnd.dp.sync()
    only(rnd.read(0, "dx"), np.s_[row, :])
    only(rnd.read(0, "dw"), np.s_[:, column])
    only(rnd.read(0, "db"), column)
    rnd.close()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,F,N", [(1, 8, 8, 8), (5, 72, 136, 40), (70, 136, 264, 520), (128, 8, 264, 264), (500, 8, 520, 72), (2048, 8, 4096, 8)])
def test_gated(M, K, F, N, act):
    rng = np.random.default_rng(M)
    jobs = [bu.gated_job(rng, M, K, F, N, act=act, train=True)]
    rnd = bu.run_gated(jobs)
    row, column = M // 2, F - 5
    gu = rnd.read(0, "gu")
    gu[row, column] = np.nan
    rnd.load(0, "gu", gu)
    grads, keep = bu.gated_grad_descs(rnd, jobs)
    assert rnd.dp.pool.grouped_gated_backward(grads, stream=rnd.dp.stream) == salus.OK
    rnd.dp.sync()
    only(rnd.read(0, "dx"), np.s_[row, :])
    only(rnd.read(0, "dw_in"), np.s_[:, [column, F + column]])
    assert np.isfinite(rnd.read(0, "dw_out")).all()
    rnd.close()
