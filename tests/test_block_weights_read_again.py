"""Weights that a backward pass reads again are not asked for non-temporally (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import pytest

from block_rounds import PAST, jobs, kernels

SIZES = [jobs(4, 128, 64, 16384, 64), jobs(4, 128, 8, 64, 32768), jobs(4, 100, 64, 16384, 16384)]


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    rounds = [(kind, s, PAST) for kind in ("gated", "gated_train") for s in SIZES]
    out = kernels(rounds, tmp_path_factory.mktemp("recorder"))
    return out[:len(SIZES)], out[len(SIZES):]


def once(names):
    return [n.endswith(", true>") for n in names if n.startswith("block_tiled")]


def test_inference_streams_them_past_the_caches(launched):
    assert [any(once(names)) for names in launched[0]] == [True] * len(SIZES), launched[0]
    assert once(launched[0][1])[-1]          # the second product


def test_training_does_not(launched):
    assert not any(any(once(names)) for names in launched[1]), launched[1]
