"""Infinite weights in the first and the last rows and columns, on the GPU: what they are no factor of is as it was, to the bit - also where a tile's lanes are
past the end of the contraction."""
import numpy as np
import pytest

import block_util as bu
from oracle import block
from paper_1902_04610_amd import salus

pytestmark = pytest.mark.gpu
SIZES = [(1, 8, 8, 8), (1, 1000, 264, 1000), (3, 2056, 136, 72), (16, 72, 520, 264), (20, 264, 72, 136), (40, 1000, 136, 72), (70, 136, 520, 264),
         (128, 72, 264, 1032), (200, 1032, 264, 264), (300, 264, 520, 136), (2048, 72, 1032, 264)]


def corners(rows, columns):
    return [(0, 0), (rows - 1, columns - 1), (rows - 1, 0), (0, columns // 2), (rows - 3, columns - 2)]


def same_but(got, clean, columns, infinite=True):
    """Columns that are infinite (or at least not finite), and all others as they were."""
    where = np.zeros(got.shape[1], bool)
    where[columns] = True
    assert np.isinf(got[:, where]).all() if infinite else not np.isfinite(got[:, where]).any()
    assert np.array_equal(got[:, ~where], clean[:, ~where])


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N,_", SIZES)
def test_dense(M, K, N, _, out):
    rng = np.random.default_rng(M + K)
    jobs = [bu.dense_job(rng, M, K, N, act=block.NONE, out=out, bias=M % 2 == 0)]
    rnd = bu.run_dense(jobs)
    clean, w = rnd.read(0, "y"), jobs[0]["parts"][2]["w"]
    descs, keep = bu.dense_descs(rnd, jobs)
    for k, n in corners(K, N):
        bad = w.copy()
        bad[k, n] = np.inf
        rnd.load(0, "w", bad)
        assert rnd.dp.pool.grouped_dense_forward(descs, stream=rnd.dp.stream) == salus.OK
        rnd.dp.sync()
        same_but(rnd.read(0, "y"), clean, [n])
    rnd.close()


@pytest.mark.parametrize("M,K,N,_", SIZES)
def test_dense_backward(M, K, N, _):
    rng = np.random.default_rng(M + K + 1)
    jobs = [bu.dense_job(rng, M, K, N, act=block.GELU, train=True)]
    rnd = bu.run_dense(jobs)
    clean = {n: rnd.read(0, n) for n in ("dx", "dw", "db")}
    w = jobs[0]["parts"][2]["w"]
    grads, keep = bu.dense_grad_descs(rnd, jobs)
    for k, n in corners(K, N):
        bad = w.copy()
        bad[k, n] = np.inf
        rnd.load(0, "w", bad)
        assert rnd.dp.pool.grouped_dense_backward(grads, stream=rnd.dp.stream) == salus.OK
        rnd.dp.sync()
        same_but(rnd.read(0, "dx"), clean["dx"], [k], False)
        assert np.array_equal(rnd.read(0, "dw"), clean["dw"]) and np.array_equal(rnd.read(0, "db"), clean["db"])
    rnd.close()


@pytest.mark.parametrize("M,K,F,N", SIZES)
def test_gated(M, K, F, N):
    rng = np.random.default_rng(M + K + 2)
    jobs = [bu.gated_job(rng, M, K, F, N, act=block.NONE)]
    rnd = bu.run_gated(jobs)
    clean = {n: rnd.read(0, n) for n in ("h", "y")}
    w_in, w_out = jobs[0]["parts"][2]["w_in"], jobs[0]["parts"][2]["w_out"]
    descs, keep = bu.gated_descs(rnd, jobs)

    def run():
        assert rnd.dp.pool.grouped_gated_forward(descs, stream=rnd.dp.stream) == salus.OK
        rnd.dp.sync()

    for k, c in corners(K, 2 * F):
        bad = w_in.copy()
        bad[k, c] = -np.inf
        rnd.load(0, "w_in", bad)
        run()
        same_but(rnd.read(0, "h"), clean["h"], [c % F])
    rnd.load(0, "w_in", w_in)
    for f, n in corners(F, N):
        bad = w_out.copy()
        bad[f, n] = np.inf
        rnd.load(0, "w_out", bad)
        run()
        assert np.array_equal(rnd.read(0, "h"), clean["h"])
        same_but(rnd.read(0, "y"), clean["y"], [n])
    rnd.close()


@pytest.mark.parametrize("M,K,F,N", SIZES)
def test_gated_backward(M, K, F, N):
    rng = np.random.default_rng(M + K + 3)
    jobs = [bu.gated_job(rng, M, K, F, N, act=block.SILU, train=True)]
    rnd = bu.run_gated(jobs)
    clean = {n: rnd.read(0, n) for n in ("dx", "dw_in", "dw_out")}
    w_in, w_out = jobs[0]["parts"][2]["w_in"], jobs[0]["parts"][2]["w_out"]
    grads, keep = bu.gated_grad_descs(rnd, jobs)

    def run():
        assert rnd.dp.pool.grouped_gated_backward(grads, stream=rnd.dp.stream) == salus.OK
        rnd.dp.sync()

    for k, c in corners(K, 2 * F):
        bad = w_in.copy()
        bad[k, c] = np.inf
        rnd.load(0, "w_in", bad)
        run()
        same_but(rnd.read(0, "dx"), clean["dx"], [k], False)
        assert np.array_equal(rnd.read(0, "dw_in"), clean["dw_in"]) and np.array_equal(rnd.read(0, "dw_out"), clean["dw_out"])
    rnd.load(0, "w_in", w_in)
    for f, n in corners(F, N):
        bad = w_out.copy()
        bad[f, n] = np.inf
        rnd.load(0, "w_out", bad)
        run()
        same_but(rnd.read(0, "dw_in"), clean["dw_in"], [f, F + f], M == 1)      # rows of both signs make a NaN
        assert np.array_equal(rnd.read(0, "dw_out"), clean["dw_out"])
    rnd.close()
