"""The rounds that reach every kernel of the transformer-block operators (test_block_dispatch.py), on the GPU against the oracle."""
import numpy as np
import pytest

import block_util as bu
from block_rounds import ROUNDS
from oracle import block
from paper_1902_04610_amd import salus

pytestmark = pytest.mark.gpu


class Repeated:
    """Normal values, a million and three of them over and over."""

    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)
        self.values = self.rng.standard_normal(1000003)

    def standard_normal(self, shape):
        n = int(np.prod(shape))
        start = int(self.rng.integers(len(self.values)))
        return np.resize(self.values[start:] if n <= len(self.values) - start else self.values, n).reshape(shape)


@pytest.mark.parametrize("number", range(len(ROUNDS)))
def test_round(number):
    kind, sizes, idle, kernels = ROUNDS[number]
    print(kind, len(sizes), "x", sizes[0], kernels, flush=True)
    rng = Repeated(number)
    train = kind.endswith("_train")
    if kind.startswith("gated"):
        jobs = [bu.gated_job(rng, *size, act=block.SILU, train=train) for size in sizes]
    elif kind.startswith("dense"):
        jobs = [bu.dense_job(rng, *size, act=block.GELU, train=train) for size in sizes]
    else:
        jobs = [bu.clip_job(rng, list(size), ["bf16"] * len(size), scale=3.0 if i % 2 == 0 else 0.5, sgd=kind == "clip_sgd") for i, size in enumerate(sizes)]
    parts = [j["parts"] for j in jobs]
    if idle:
        other = bu.Buffers()
        other.add("idle", (idle,), "raw")
        parts.append((other, bu.Buffers(), {}, []))
    rnd = bu.Round(parts)
    pool = rnd.dp.pool

    def call(run, made):
        descs, keep = made
        assert run(descs, stream=rnd.dp.stream) == salus.OK, pool.last_error()

    if kind.startswith("gated"):
        call(pool.grouped_gated_forward, bu.gated_descs(rnd, jobs))
        if train:
            call(pool.grouped_gated_backward, bu.gated_grad_descs(rnd, jobs))
        rnd.dp.sync()
        bu.check_gated(rnd, jobs)
    elif kind.startswith("dense"):
        call(pool.grouped_dense_forward, bu.dense_descs(rnd, jobs))
        if train:
            call(pool.grouped_dense_backward, bu.dense_grad_descs(rnd, jobs))
        rnd.dp.sync()
        bu.check_dense(rnd, jobs)
    else:
        call(pool.grouped_clip_sgd if kind == "clip_sgd" else pool.grouped_clip, bu.clip_descs(rnd, jobs))
        rnd.dp.sync()
        bu.check_clip(rnd, jobs)
    rnd.close()
