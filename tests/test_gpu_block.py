"""Transformer-block operators on the GPU against the oracle in 64 bits: sizes from one row to many, odd widths, rounds of one job and
of more than a launch holds, every activation, with and without residual, bias and what the backward pass needs."""
import numpy as np
import pytest
import torch

import block_util as bu
from oracle import block
from paper_1902_04610_amd import salus

pytestmark = pytest.mark.gpu
ACTS = [block.NONE, block.RELU, block.GELU, block.SILU]

SIZES = [  # M, K, F, N
    (1, 8, 8, 8), (1, 64, 128, 64), (1, 1024, 1024, 1024), (2, 200, 40, 72), (3, 72, 264, 24), (7, 1000, 136, 1000), (15, 136, 8, 264), (16, 64, 64, 64),
    (17, 520, 72, 8), (31, 264, 520, 136), (32, 1024, 256, 128), (33, 40, 136, 200), (63, 128, 128, 128), (64, 320, 64, 1032), (65, 8, 328, 64),
    (127, 72, 72, 72), (128, 512, 256, 512), (129, 264, 136, 72), (192, 128, 512, 256), (257, 136, 264, 520), (300, 1000, 200, 136), (600, 64, 1000, 72),
]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_gated_sizes(size):
    M, K, F, N = size
    rng = np.random.default_rng(M * 7 + K)
    jobs = [bu.gated_job(rng, M, K, F, N, act=ACTS[(M + K) % 4], residual=M % 3 != 0)]
    rnd = bu.run_gated(jobs)
    bu.check_gated(rnd, jobs)
    rnd.close()


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_gated_training_sizes(size):
    M, K, F, N = size
    rng = np.random.default_rng(M * 7 + K + 1)
    jobs = [bu.gated_job(rng, M, K, F, N, act=ACTS[(M + K + 1) % 4], residual=M % 3 != 0, train=True)]
    rnd = bu.run_gated(jobs)
    bu.check_gated(rnd, jobs)
    rnd.close()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("train", [False, True])
def test_gated_activations_far_out(act, train):
    """Gates from far below to far above the bend."""
    rng = np.random.default_rng(act)
    jobs = [bu.gated_job(rng, 40, 64, 96, 72, act=act, train=train, scale=s) for s in (0.01, 1.0, 8.0)]
    rnd = bu.run_gated(jobs)
    bu.check_gated(rnd, jobs)
    rnd.close()


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_dense_sizes(size, out):
    M, K, N, _ = size
    rng = np.random.default_rng(M * 11 + K)
    jobs = [bu.dense_job(rng, M, K, N, act=ACTS[(M + K) % 4], out=out, bias=M % 2 == 0, residual=M % 3 != 0)]
    rnd = bu.run_dense(jobs)
    bu.check_dense(rnd, jobs)
    rnd.close()


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_dense_training_sizes(size):
    M, K, N, _ = size
    rng = np.random.default_rng(M * 13 + K)
    jobs = [bu.dense_job(rng, M, K, N, act=ACTS[(M + K + 1) % 4], bias=M % 4 != 1, residual=M % 3 != 0, train=True)]
    rnd = bu.run_dense(jobs)
    bu.check_dense(rnd, jobs)
    rnd.close()


@pytest.mark.parametrize("rows", [(1, 5), (1, 32), (20, 130), (1, 400)], ids=str)
@pytest.mark.parametrize("train", [False, True])
def test_mixed_rounds(rows, train):
    """Jobs of different sizes in one call; every other option differs between neighbours."""
    rng = np.random.default_rng(rows[1])
    pick = lambda: int(rng.integers(rows[0], rows[1] + 1))
    width = lambda: 8 * int(rng.integers(1, 60))
    gated = [bu.gated_job(rng, pick(), width(), width(), width(), act=ACTS[i % 4], residual=i % 2 == 0, in_place=i % 4 == 2, train=train) for i in range(9)]
    rnd = bu.run_gated(gated)
    bu.check_gated(rnd, gated)
    rnd.close()
    dense = [bu.dense_job(rng, pick(), width(), width(), act=ACTS[i % 4], out="bf16" if train or i % 3 else "f32", bias=i % 2 == 0, residual=i % 4 < 2,
                          in_place=i % 3 == 1 and i % 4 < 2, train=train) for i in range(9)]
    rnd = bu.run_dense(dense)
    bu.check_dense(rnd, dense)
    rnd.close()


def test_more_jobs_than_a_launch_holds():
    rng = np.random.default_rng(8)
    jobs = [bu.gated_job(rng, 1 + i % 5, 16, 8 + 8 * (i % 3), 24, act=ACTS[i % 4], train=True) for i in range(70)]
    rnd = bu.run_gated(jobs)
    bu.check_gated(rnd, jobs)
    rnd.close()
    jobs = [bu.dense_job(rng, 1 + i % 20, 16, 8 + 8 * (i % 3), act=ACTS[i % 4], train=True) for i in range(70)]
    rnd = bu.run_dense(jobs)
    bu.check_dense(rnd, jobs)
    rnd.close()


def test_gradients_of_the_input_can_be_left_out():
    rng = np.random.default_rng(9)
    jobs = [bu.gated_job(rng, 20, 64, 40, 24, train=True)]
    rnd = bu.run_gated(jobs)
    before = rnd.read(0, "dx")
    rnd.load(0, "dx", np.full((20, 64), 7.0))
    descs, keep = bu.gated_grad_descs(rnd, jobs, dx=False)
    assert rnd.dp.pool.grouped_gated_backward(descs, stream=rnd.dp.stream) == salus.OK
    rnd.dp.sync()
    assert (rnd.read(0, "dx") == 7.0).all() and np.isfinite(before).all()
    rnd.close()


@pytest.mark.parametrize("M", [1, 20, 70, 200])
def test_what_is_not_finite_stays_in_its_row(M):
    """A NaN and an infinity in one row of X: that row of Y is not finite, all others are as they were."""
    rng = np.random.default_rng(M)
    jobs = [bu.gated_job(rng, M, 72, 40, 136, act=block.SILU)]
    clean = bu.run_gated(jobs)
    y = clean.read(0, "y")
    clean.close()
    row = M // 2
    jobs[0]["parts"][2]["x"][row, 5] = np.nan
    jobs[0]["parts"][2]["x"][row, 70] = np.inf
    rnd = bu.run_gated(jobs)
    got = rnd.read(0, "y")
    rnd.close()
    assert np.isnan(got[row]).all()
    assert np.array_equal(np.delete(got, row, 0), np.delete(y, row, 0))
    for act in ACTS:
        jobs = [bu.dense_job(rng, M, 72, 136, act=act, out="f32")]
        jobs[0]["parts"][2]["x"][row, 71] = np.nan
        rnd = bu.run_dense(jobs)
        got = rnd.read(0, "y")
        rnd.close()
        assert np.isnan(got[row]).all() and np.isfinite(np.delete(got, row, 0)).all()


@pytest.mark.parametrize("sgd", [False, True])
@pytest.mark.parametrize("counts,dtypes", [
    ([1], ["f32"]), ([1], ["bf16"]), ([7, 9, 1], ["bf16", "f32", "bf16"]), ([4096], ["f32"]), ([4097, 4095, 8, 1001], ["bf16", "bf16", "f32", "bf16"]),
    ([100003, 17, 65536], ["f32", "bf16", "bf16"]), ([5000000], ["bf16"]), ([33] * 130, ["bf16", "f32"] * 65),
], ids=str)
def test_clip(counts, dtypes, sgd):
    rng = np.random.default_rng(len(counts) + sum(counts))
    # norms of about 5, 0.5 (nothing to scale) and exactly zero
    jobs = [bu.clip_job(rng, counts, dtypes, scale=s, sgd=sgd, max_norm=m) for s, m in ((5.0, 1.0), (0.5, 1.0), (0.0, 1.0), (5.0, np.inf))]
    rnd = bu.run_clip(jobs)
    bu.check_clip(rnd, jobs)
    rnd.close()


def test_clip_of_many_jobs():
    rng = np.random.default_rng(4)
    jobs = [bu.clip_job(rng, [1 + 13 * i, 5 + i], ["bf16", "f32"], scale=0.5 + i % 7, sgd=True, lr=0.01 * i) for i in range(70)]
    rnd = bu.run_clip(jobs)
    bu.check_clip(rnd, jobs)
    rnd.close()


def test_clip_of_what_is_not_finite():
    """An infinite gradient: coefficient zero, itself NaN; a NaN: everything NaN.  Squares beyond the largest float are no infinity."""
    rng = np.random.default_rng(5)
    jobs = [bu.clip_job(rng, [40, 3000], ["f32", "bf16"], scale=5.0) for _ in range(3)]
    jobs[0]["parts"][2]["g0"][3] = np.inf
    jobs[1]["parts"][2]["g1"][2999] = np.nan
    jobs[2]["parts"][2]["g0"][:] = np.float32(1e30)
    rnd = bu.run_clip(jobs)
    assert rnd.read(0, "norm")[0] == np.inf and np.isnan(rnd.read(0, "g0")[3]) and (np.delete(rnd.read(0, "g0"), 3) == 0).all() and (rnd.read(0, "g1") == 0).all()
    assert np.isnan(rnd.read(1, "norm")[0]) and np.isnan(rnd.read(1, "g0")).all() and np.isnan(rnd.read(1, "g1")).all()
    assert abs(rnd.read(2, "norm")[0] / (1e30 * np.sqrt(40)) - 1) < 1e-6 and abs(rnd.read(2, "g0")[0] * np.sqrt(40) - 1) < 1e-6
    rnd.close()


def test_clip_without_a_limit_leaves_infinities():
    rng = np.random.default_rng(10)
    jobs = [bu.clip_job(rng, [40, 3000], ["f32", "bf16"], scale=5.0, max_norm=np.inf) for _ in range(2)]
    jobs[0]["parts"][2]["g0"][3] = np.inf
    jobs[1]["parts"][2]["g0"][3] = np.nan
    rnd = bu.run_clip(jobs)
    assert rnd.read(0, "norm")[0] == np.inf and all(np.array_equal(rnd.read(0, n), jobs[0]["parts"][2][n]) for n in ("g0", "g1"))
    assert np.isnan(rnd.read(1, "norm")[0]) and np.isnan(rnd.read(1, "g0")).all()
    rnd.close()


def test_the_same_bits_every_time_and_on_another_stream():
    rng = np.random.default_rng(6)
    gated = [bu.gated_job(rng, m, 264, 136, 200, train=True) for m in (1, 40, 150)]
    clips = [bu.clip_job(rng, [50000, 333], ["bf16", "f32"], scale=3.0, sgd=True)]
    side = torch.cuda.Stream()
    names = ["y", "h", "gu", "dx", "dw_in", "dw_out"]
    results = []
    for stream in (None, side.cuda_stream, None):
        rnd = bu.run_gated(gated, stream)
        results.append([rnd.read(i, n) for i in range(3) for n in names])
        rnd.close()
        rnd = bu.run_clip(clips, stream)
        results[-1] += [rnd.read(0, n) for n in ("norm", "wm0", "wm1")]
        rnd.close()
    for other in results[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(results[0], other))


def test_a_recorded_step_replays_with_new_inputs():
    """Forward, backward and clipped update in one graph; between the replays eager work on other data of the same jobs."""
    rng = np.random.default_rng(7)
    M, K, F, N = 24, 72, 136, 72
    job = bu.gated_job(rng, M, K, F, N, train=True)
    p, l, d, written = job["parts"]
    counts = [K * 2 * F, F * N]
    for t, (n, name) in enumerate(zip(counts, ("w_in", "w_out"))):
        p.add(f"wm{t}", (n,), "f32")
        d[f"wm{t}"] = d[name].reshape(-1)
    l.add("norm", (1,), "f32")
    l.add("clip_work", (salus.clip_work_bytes([dict(g_off=0, count=n, dtype=0) for n in counts]),), "raw")
    rnd = bu.Round([job["parts"]])
    pool = rnd.dp.pool
    fwd, k1 = bu.gated_descs(rnd, [job])
    bwd, k2 = bu.gated_grad_descs(rnd, [job])
    o = {k: v[0] for k, v in {**p.at, **l.at}.items()}
    clip, k3 = salus.Pool.make_clip_descs([dict(job=rnd.ids[0], max_norm=0.01, lr=0.5, norm_off=o["norm"], work_off=o["clip_work"], tensors=[
        dict(g_off=o["dw_in"], count=counts[0], dtype=salus.BF16, wm_off=o["wm0"], wb_off=o["w_in"]),
        dict(g_off=o["dw_out"], count=counts[1], dtype=salus.BF16, wm_off=o["wm1"], wb_off=o["w_out"])])])

    def step(stream):
        assert pool.grouped_gated_forward(fwd, stream=stream) == salus.OK
        assert pool.grouped_gated_backward(bwd, stream=stream) == salus.OK
        assert pool.grouped_clip_sgd(clip, stream=stream) == salus.OK

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side.cuda_stream)
    names = ["y", "dx", "dw_in", "dw_out", "norm", "wm0", "wm1", "w_in", "w_out"]
    for turn in range(4):
        x, dy = bu.bf16(rng.standard_normal((M, K))), bu.bf16(rng.standard_normal((M, N)))
        results = []
        for replay in (False, True):
            rnd.restore()
            rnd.load(0, "x", x)
            rnd.load(0, "dy", dy)
            torch.cuda.synchronize()
            graph.replay() if replay else step(rnd.dp.stream)
            torch.cuda.synchronize()
            results.append([rnd.read(0, n) for n in names])
        assert all(np.array_equal(a, b) for a, b in zip(*results)), turn
        assert np.isfinite(results[0][0]).all() and results[0][4][0] > 0.01
    rnd.close()
