"""How input and weight gradients share a launch of more tiles than it has workgroups (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import pytest

from block_launches import launches
from block_splits import SPLITS


@pytest.fixture(scope="module")
def recorded(tmp_path_factory):
    return launches([s[:2] + (0,) for s in SPLITS], tmp_path_factory.mktemp("recorder"))


def tiles(kind, sizes):
    up = lambda v: -(-v // 128)
    x = sum(up(s[0]) * up(s[1]) for s in sizes)
    if kind == "dense_train":
        return x, sum(up(K) * up(N) for _, K, N in sizes)
    return x, sum(up(K) * up(2 * F) + up(F) * up(N) for _, K, F, N in sizes)


@pytest.mark.parametrize("number", range(len(SPLITS)))
def test_places(recorded, number):
    kind, sizes, want = SPLITS[number]
    shared = [l for l in recorded[number] if l.kernel == "gradients_tiled"]
    assert len(shared) == 1 and shared[0].words[:3] == want, recorded[number]
    sums, inputs, weights = want
    assert shared[0].grid == sums + inputs + weights and inputs + weights <= 512
    x, w = tiles(kind, sizes)
    assert x + w > 512 and inputs <= x and weights < w and sums % 8 == 0
