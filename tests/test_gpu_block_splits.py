"""Input and weight gradients (and bias gradients) that share a launch and walk several tiles each, on the GPU against the oracle."""
import pytest

import block_util as bu
from block_splits import SPLITS
from oracle import block
from test_gpu_block_rounds import Repeated

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("number", range(len(SPLITS)))
def test_split(number):
    kind, sizes, _ = SPLITS[number]
    print(kind, len(sizes), "x", sizes[0], flush=True)
    rng = Repeated(100 + number)
    if kind == "gated_train":
        jobs = [bu.gated_job(rng, *size, act=[block.GELU, block.SILU][i % 2], train=True) for i, size in enumerate(sizes)]
        rnd = bu.run_gated(jobs)
        bu.check_gated(rnd, jobs)
    else:
        jobs = [bu.dense_job(rng, *size, act=[block.GELU, block.RELU][i % 2], train=True) for i, size in enumerate(sizes)]
        rnd = bu.run_dense(jobs)
        bu.check_dense(rnd, jobs)
    rnd.close()
