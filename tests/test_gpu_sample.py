"""Sampling against the oracle: every token is the same."""
import numpy as np
import pytest

from answer_util import Round, check_sample, sample_descs, sample_job
from oracle import answer
from paper_1902_04610_amd import salus, synth

pytestmark = pytest.mark.gpu


def run(jobs):
    r = Round([(p, l) for p, l, _ in jobs])
    descs, keep = sample_descs(r, jobs)
    assert r.dp.pool.grouped_sample(descs, stream=r.dp.stream) == salus.OK, r.dp.pool.last_error()
    r.dp.sync()
    check_sample(r, jobs)
    r.check_rest("tokens", "work")
    r.close()


def to_bf16(x):
    return answer.bf16_values(synth.f32_to_bf16_bits(x.astype(np.float32))).astype(np.float32)


def logits(rng, M, V, kind):
    x = rng.standard_normal((M, V)) * 2
    if kind == "peaked":
        for row in x:
            row[rng.integers(0, V, 12)] += rng.uniform(4, 12, 12)
    if kind == "equal":
        x[:] = 1.5
    if kind == "ties":
        x = np.round(x)
    if kind == "masked":
        x[rng.random((M, V)) < 0.9] = -np.inf
        x[:, V // 2] = 0
    return x.astype(np.float32)


def limits(rng, M):
    """Every combination of limits comes up."""
    out = []
    for i in range(M):
        out.append((float(rng.choice([0.5, 1.0, 1.7])), int(rng.integers(2, 300)) if i & 1 else 0, float(rng.uniform(0.3, 0.99)) if i & 2 else 1.0,
                    float(rng.uniform(0.001, 0.3)) if i & 4 else 0.0))
    return out


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("kind", ["flat", "peaked", "equal", "ties", "masked"])
@pytest.mark.parametrize("V", [1, 7, 64, 1000, 4096, 50257])
def test_all_limits(V, kind, bf16):
    rng = np.random.default_rng(V)
    M = 16 if V < 5000 else 8
    x = logits(rng, M, V, kind)
    run([sample_job(to_bf16(x) if bf16 else x, limits(rng, M), rng.uniform(0.0001, 0.9999, M), bf16, pad=8 * (V % 3))])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", [1100, 2597, 3100, 4099, 8200])
def test_rows_that_fill_only_some_of_their_runs(V, bf16):
    """Flat rows whose kept tokens no list holds; random numbers up to the last of them."""
    rng = np.random.default_rng(V)
    x = (rng.standard_normal((64, V)) * 1.5).astype(np.float32)
    limits = [(1.0, 0, 1.0, 0.01), (1.1, 0, 0.95, 0.01), (1.0, 600, 0.9, 0.0), (0.9, 500, 1.0, 0.02)]
    run([sample_job(to_bf16(x) if bf16 else x, limits * 16, (np.arange(64) // 4 + 0.99) / 16, bf16)])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", [900, 2597, 20011])
def test_where_top_p_ends(V, bf16):
    """One row after the other, behind top_k and alone: the last kept token and the first that is not differ by any of a place's bits."""
    rng = np.random.default_rng(V)
    x = (rng.standard_normal((96, V)) * 1.5).astype(np.float32)
    limits = [(float(rng.uniform(0.6, 1.2)), 0 if i % 2 else int(rng.integers(20, 200)), float(rng.uniform(0.5, 0.97)), 0.0) for i in range(96)]
    run([sample_job(to_bf16(x) if bf16 else x, limits, rng.choice([0.2, 0.5, 0.9, 0.97, 0.995, 0.9999], 96), bf16)])


def test_top_p_ends_in_front_of_thousands_of_almost_equal_logits():
    """Three kept tokens, the last a few float steps above 3000 equal ones, next to multiples of 1 / 16 of a power of two."""
    rng = np.random.default_rng(3)
    rows, limits, V = [], [], 3100
    for n in range(30, 70):
        edge = np.float32(n) / (np.float32(16.0) * np.float32(1.4426950))
        step = np.spacing(edge)
        x = np.full(V, -20.0, np.float32)
        x[rng.permutation(V)[:3003]] = edge - 2 * step
        three = rng.permutation(np.nonzero(x > 0)[0])[:3]
        x[three] = edge + np.float32(1.5), edge + np.float32(0.02), edge + 4 * step
        w = np.exp(x.astype(np.float64) - x.max())
        rows.append(x)
        limits.append((1.0, 0, float((w[three[:2]].sum() + 0.5 * w[three[2]]) / w.sum()), 0.0))
    run([sample_job(np.array(rows), limits, rng.uniform(0.02, 0.98, len(rows)))])


@pytest.mark.parametrize("V,M", [(131072, 3), (200003, 2), (524288, 1)])
def test_large_vocabularies(V, M):
    rng = np.random.default_rng(V)
    run([sample_job(logits(rng, M, V, "flat"), [(1.0, 0, 0.9, 0.0), (0.8, 5000, 0.95, 0.0), (1.2, 0, 1.0, 0.0)][:M], rng.uniform(0, 1, M))])


def test_rows_that_hold_no_numbers():
    rng = np.random.default_rng(1)
    x = logits(rng, 12, 300, "flat")
    x[0] = np.nan
    x[1] = -np.inf
    x[2, :] = -np.inf
    x[2, 77] = -3e38
    x[3, ::2] = np.nan
    x[4, [5, 200]] = np.inf
    x[5] = np.finfo(np.float32).min
    x[6, 10] = np.finfo(np.float32).max
    x[7, :] = [0.0, -0.0] * 150
    x[8, 3] = np.inf
    x[8, 2] = np.nan
    x[9] = 1e-42
    p = [(1.0, 0, 1.0, 0.0)] * 12
    p[3], p[5], p[7], p[9], p[10], p[11] = (1.0, 20, 0.9, 0.01), (1.0, 5, 1.0, 0.0), (1.0, 7, 1.0, 0.0), (1.0, 0, 0.5, 0.0), (1e-30, 0, 1.0, 0.0), (1e30, 0, 0.5, 0.2)
    run([sample_job(x, p, rng.uniform(0.01, 0.99, 12)), sample_job(to_bf16(x), p, rng.uniform(0.01, 0.99, 12), True)])


def test_parameters_out_of_range():
    rng = np.random.default_rng(2)
    x = logits(rng, 12, 500, "peaked")
    nan = float("nan")
    p = [(0.0, 0, 1.0, 0.0), (-1.0, 9, 0.5, 0.5), (nan, 0, 1.0, 0.0), (1.0, -3, 1.0, 0.0), (1.0, 10 ** 9, 1.0, 0.0), (1.0, 0, -1.0, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 2.0, 0.0),
         (1.0, 0, 1.0, 5.0), (1.0, 1, 0.5, 0.1), (1.0, 0, nan, nan), (1.0, 0, 1.0, -1.0)]
    run([sample_job(x, p, rng.uniform(0.01, 0.99, 12))])
    run([sample_job(x, [(1.0, 40, 1.0, 0.0)] * 12, [0.0, 1.0, 2.0, -1.0, nan, 0.99999994, 1e-30, 0.5, 0.25, 0.75, 0.1, 0.9])])


def test_the_share_of_every_token():
    """Evenly spread numbers give every token as often as its weight says, to within one."""
    M, V = 4096, 50
    x = np.tile(np.linspace(-1, 1, V, dtype=np.float32), (M, 1))
    u = (np.arange(M) + 0.5) / M
    jobs = [sample_job(x, [(1.0, 0, 1.0, 0.0)] * M, u)]
    r = Round([(p, l) for p, l, _ in jobs])
    descs, keep = sample_descs(r, jobs)
    assert r.dp.pool.grouped_sample(descs, stream=r.dp.stream) == salus.OK
    r.dp.sync()
    w = np.exp(x[0].astype(np.float64))
    assert np.abs(np.bincount(r.read(0, "tokens"), minlength=V) - M * w / w.sum()).max() <= 1
    r.close()


@pytest.mark.parametrize("count", [3, 30])
def test_jobs_of_many_kinds_together(count):
    rng = np.random.default_rng(count)
    jobs = []
    for j in range(count):
        M, V = 1 + j % 5, 100 + 777 * j
        x = logits(rng, M, V, ("flat", "peaked", "ties")[j % 3])
        jobs.append(sample_job(to_bf16(x) if j % 2 else x, limits(rng, M), rng.uniform(0.001, 0.999, M), j % 2 == 1))
    run(jobs)
