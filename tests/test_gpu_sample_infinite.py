"""Sampling of rows that hold infinite logits, or the largest floats, behind every limit: every token is the oracle's."""
import numpy as np
import pytest

from answer_util import Round, check_sample, sample_descs, sample_job
from oracle import answer
from paper_1902_04610_amd import salus, synth

pytestmark = pytest.mark.gpu
LARGEST = np.finfo(np.float32).max

# top_k, top_p, min_p
LIMITS = [(0, 1.0, 0.05), (0, 1.0, 1.0), (0, 1.0, 1e-30), (0, 1.0, 1e-45), (2, 1.0, 0.05), (5, 1.0, 1.0), (40, 1.0, 0.3), (300, 1.0, 0.01), (0, 0.5, 0.05), (0, 0.9, 1.0), (0, 0.99, 1e-30),
          (5, 0.5, 0.05), (300, 0.9, 0.3), (0, 0.9, 0.0), (5, 1.0, 0.0), (40, 0.7, 0.0), (0, 1.0, 0.0)]


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


def places(rng, V, where):
    return {"one": [V // 3], "one slice": sorted(rng.permutation(min(V, 900))[:7]), "all over": sorted(rng.permutation(V)[:9]), "first and last": [0, V - 1],
            "more than lists hold": sorted(rng.permutation(V)[:max(2, 3 * V // 4)])}[where]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("where", ["one", "one slice", "all over", "first and last", "more than lists hold"])
@pytest.mark.parametrize("V", [300, 8192, 20003, 50257])
def test_infinite_logits_behind_every_limit(V, where, bf16):
    rng = np.random.default_rng(V)
    x = (rng.standard_normal((2 * len(LIMITS), V)) * 2).astype(np.float32)
    x[:, 17::31] = np.nan
    x[:, 5::40] = -np.inf
    for row in x:
        row[places(rng, V, where)] = np.inf
    # random numbers in the middle of a token's share: shares are equal, and no sum's rounding reaches a border
    u = [(int(v) + 0.5) / len(places(rng, V, where)) for v in rng.integers(0, len(places(rng, V, where)), len(x))]
    run([sample_job(to_bf16(x) if bf16 else x, [(T, *l) for T in (1.0, 0.01) for l in LIMITS], u, bf16)])


@pytest.mark.parametrize("V", [300, 9001])
@pytest.mark.parametrize("temperature", [1e-38, 1e-3, 1.0, 1e30, 3e38])
def test_the_largest_and_smallest_floats_behind_every_limit(temperature, V):
    """Where top + temperature ln min_p, or its margin, is beyond what a float holds."""
    rng = np.random.default_rng(V)
    kinds = []
    for fill, top in ((0.0, LARGEST), (-LARGEST, -LARGEST), (-LARGEST, LARGEST), (-np.inf, -LARGEST), (-1e-45, 1e-45), (0.0, 0.0), (-np.inf, 1e30)):
        x = np.full((len(LIMITS), V), fill, np.float32)
        x[:, [V // 5, V // 2]] = top
        kinds.append(sample_job(x, [(temperature, *l) for l in LIMITS], rng.choice([0.2501, 0.4999, 0.7499], len(LIMITS))))
    run(kinds)
