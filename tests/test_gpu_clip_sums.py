"""Sums of squares whose terms differ by more than a float holds, on the GPU: the norm is the 64-bit sum's, rounded once."""
import numpy as np
import pytest

import block_util as bu
from oracle import block

pytestmark = pytest.mark.gpu

# 255 / 128 . 2^-13: its square is 0.992 . 2^-24, which a float sum of 1 and more loses; seven of them are 3.5 half steps of the norm
SMALL = 255 / 128 * 2.0 ** -13


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("place", [0, 3, 7])
@pytest.mark.parametrize("count", [8, 8 * 300, 3 * 4096, 2500 * 4096 + 8 * 5])
def test_one_large_and_seven_small(count, place, dtype):
    g = np.full(count, SMALL)
    g[place::8] = 1.0
    job = bu.clip_job(np.random.default_rng(0), [count], [dtype], max_norm=np.inf)
    job["parts"][2]["g0"] = g
    rnd = bu.run_clip([job])
    got = rnd.read(0, "norm")[0]
    rnd.close()
    norm = np.sqrt(count / 8 * (1 + 7 * SMALL ** 2))
    assert abs(got - norm) <= block.STEP * norm * (1 + 1e-6), (got, norm, (got / norm - 1) / block.STEP)


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -40, 1.0, 2.0 ** 40, 2.0 ** 60])
def test_bf16_over_the_range(scale):
    rng = np.random.default_rng(1)
    job = bu.clip_job(rng, [70001], ["bf16"], max_norm=np.inf, scale=scale)
    rnd = bu.run_clip([job])
    got = rnd.read(0, "norm")[0]
    rnd.close()
    norm = np.sqrt((job["parts"][2]["g0"] ** 2).sum())
    assert abs(got - norm) <= block.STEP * norm * (1 + 1e-6), (got, norm)
