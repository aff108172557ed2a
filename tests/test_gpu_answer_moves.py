"""Jobs whose caches leave the device, come back and slide down go on answering as if they had stayed."""
import numpy as np
import pytest

from paper_1902_04610_amd import salus
from test_gpu_answering import SHAPES, Answering, steps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("limit", [200, 2000])
def test_evicted_restored_and_compacted_between_steps(limit):
    rng = np.random.default_rng(limit)
    model = Answering(rng, SHAPES, 16, limit)
    r, places = model.r, set()
    for turn, new in enumerate(steps(rng, model, 7)):
        if turn:
            held = [(r.read(j, "k"), r.read(j, "v")) for j in range(3)]
            out = (turn - 1) % 3
            assert r.dp.pool.switch_out(r.ids[out]) == salus.OK, r.dp.pool.last_error()
            if turn > 1:
                r.dp.pool.compact()
            assert r.dp.pool.switch_in(r.ids[out]) == salus.OK, r.dp.pool.last_error()
            r.dp.sync()
            assert all(np.array_equal(r.read(j, name), a) for j in range(3) for name, a in zip("kv", held[j]))
        places.add(tuple(r.dp.pool.job_query(j).persist_off for j in r.ids))
        for j in range(3):
            r.write(j, "table", r.jobs[j][1]["table"])          # a lane holds nothing between iterations
        model.load(rng, new)
        before = [(r.read(j, "k"), r.read(j, "v")) for j in range(3)]
        model.call(r.dp.stream)
        r.dp.sync()
        model.check(before)
    assert len(places) > 2
    r.close()
