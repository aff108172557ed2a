"""Grids of the transformer-block kernels for the longest rounds (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import pytest

from block_launches import launches

# Rows that make more tiles than a grid of 256 threads each may have workgroups: the slopes' of 16 rows, the gate gradients' of 32
ROUNDS = [("dense_train", [((1 << 28) + 40, 8, 8)], 0), ("dense_train", [((1 << 28) + 40, 8, 8), (33, 8, 520), ((1 << 27) + 7, 8, 16)], 0),
          ("gated_train", [((1 << 29) + 40, 8, 8, 8)], 0), ("gated_train", [((1 << 31) - 1, 8, 8, 8)], 0), ("dense_train", [((1 << 31) - 1, 8, 8)], 0),
          ("gated", [((1 << 31) - 1, 8, 16, 8)], 0), ("dense", [((1 << 31) - 1, 16, 8)], 0)]


@pytest.mark.parametrize("number", range(len(ROUNDS)))
def test_a_grid_has_fewer_than_2_to_the_32_threads(number, tmp_path):
    out = launches(ROUNDS[number:number + 1], tmp_path)[0]
    assert out
    wrong = [l for l in out if l.grid * l.block >= 1 << 32]
    assert not wrong, wrong
