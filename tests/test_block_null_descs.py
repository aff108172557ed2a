"""No descriptors at all, of however many: an invalid argument, before anything is allocated for them (CPU only, a pool without device memory)."""
import pytest

from paper_1902_04610_amd import salus

CALLS = ["gated_forward", "gated_backward", "dense_forward", "dense_backward", "clip", "clip_sgd"]


@pytest.mark.parametrize("call", CALLS)
def test_null_descriptors(call):
    pool = salus.Pool(None, 1 << 20)
    run = getattr(salus.lib(), "salus_grouped_" + call)
    for n in (1, 1 << 20, 2 ** 32 - 1):
        assert run(pool._h, None, n, None) == salus.EINVAL, n
        assert "null descriptor array" in pool.last_error()
    assert run(pool._h, None, 0, None) == salus.OK
    assert run(None, None, 1, None) == salus.EINVAL
    pool.close()
