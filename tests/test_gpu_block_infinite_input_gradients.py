"""Infinite weights of input gradients whose width ends inside a k-step, on the GPU, in rounds that the narrow and the wide register tiles of transposed weights
take: the infinity that they make, in its column alone."""
import numpy as np
import pytest

import block_util as bu
from oracle import block
from paper_1902_04610_amd import salus

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_jobs,M,K,N", [(1, 16, 1032, 4104), (40, 5, 8, 72), (40, 16, 520, 72), (40, 20, 64, 72), (40, 24, 520, 72), (60, 48, 128, 8)])
def test_input_gradient(n_jobs, M, K, N):
    rng = np.random.default_rng(N)
    jobs = [bu.dense_job(rng, M, K, N, act=block.GELU, train=True) for _ in range(n_jobs)]
    rnd = bu.run_dense(jobs)
    which = (0, n_jobs - 1)
    clean = [rnd.read(i, "dx") for i in which]
    grads, keep = bu.dense_grad_descs(rnd, jobs)
    for k, n in ((0, 0), (K - 1, 0), (K - 3, 5), (1, N - 1)):
        for i in which:
            bad = jobs[i]["parts"][2]["w"].copy()
            bad[k, n] = np.inf
            rnd.load(i, "w", bad)
        assert rnd.dp.pool.grouped_dense_backward(grads, stream=rnd.dp.stream) == salus.OK
        rnd.dp.sync()
        for i, was in zip(which, clean):
            got = rnd.read(i, "dx")
            assert np.isinf(got[:, k]).all(), (i, k, n, got[:4, k])
            assert np.array_equal(np.delete(got, k, 1), np.delete(was, k, 1)), (i, k, n)
    rnd.close()
