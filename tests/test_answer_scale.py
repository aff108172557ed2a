"""Which scales of attention are taken (CPU only)."""
import numpy as np
import pytest

from paper_1902_04610_amd import salus
from test_answer_grids import CACHED, call


@pytest.mark.parametrize("scale,taken", [(2.3e38, True), (2.358e38, True), (2.3595e38, False), (float(np.finfo(np.float32).max), False), (1e-45, True)])
def test_a_scale_times_log2_e_is_a_float(scale, taken, tmp_path):
    """Scores count in powers of two: where their scale is infinite a score of zero would be no number."""
    rc, error, lines = call(tmp_path, "attention", 1, dict(CACHED, M=1, n_seqs=1, Hq=1, Hkv=1, D=32, scale=scale))
    assert (rc == salus.OK and lines) if taken else (rc == salus.EINVAL and "scale" in error and not lines)
