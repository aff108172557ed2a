"""Rounds with more tiles than one launch takes (2^23 of 16 or 32 rows), on the GPU: rows around both ends and around the seam against the oracle, and nothing
of the work buffer, NaNs before the call, left as it was."""
import numpy as np
import pytest
import torch

import block_util as bu
from oracle import block
from paper_1902_04610_amd import salus
from test_gpu_block_large import Job

pytestmark = pytest.mark.gpu


def seam(M, rows):
    """Rows at both ends and around the seam."""
    return sorted({0, 1, 31, M - 1, M - 2, M // 2} | {rows + d for d in (-33, -1, 0, 1, 33)})


def spoil(j, nbytes):
    at = j.dp.pool.job_query(j.job).lane_off + j.offsets["work_off"]
    j.dp.buf[at:at + nbytes].fill_(0xff)


def prepare(j, at, N, seed):
    dy = bu.bf16(np.random.default_rng(seed).standard_normal((len(at), N)))
    j.t["dy"][torch.as_tensor(at, device="cuda")] = torch.from_numpy(dy).to("cuda", torch.bfloat16)
    return dy


def zero_elsewhere(t, at):
    """All rows but those are zero (their dY is)."""
    t = t.clone()
    t[torch.as_tensor(at, device="cuda")] = 0
    return bool((t == 0).all())


def test_slopes():
    M, K, N = (1 << 27) + 40, 8, 8
    made = bu.Buffers(), bu.Buffers(), {}, []
    for name, shape in (("w", (K, N)), ("b", (N,))):
        made[0].add(name, shape, "bf16")
    work = salus.dense_grad_work_bytes(M, N)
    for name, shape, dtype in (("x", (M, K), "bf16"), ("y", (M, N), "bf16"), ("z", (M, N), "f32"), ("dy", (M, N), "bf16"), ("dx", (M, K), "bf16"),
                               ("dw", (K, N), "bf16"), ("db", (N,), "f32"), ("work", (work,), "raw")):
        made[1].add(name, shape, dtype)
    j = Job(made, dict(w=0.35, b=0.5, x=1.0))
    spoil(j, work)
    at = seam(M, 1 << 27)
    dy = prepare(j, at, N, 1)
    size = dict(M=M, K=K, N=N, act=salus.ACT_SILU)
    print("forward", flush=True)
    j.call(j.dp.pool.make_dense_descs, j.dp.pool.grouped_dense_forward, "w b x y z", y_dtype=salus.BF16, **size)
    j.dp.sync()
    print("backward", flush=True)
    j.call(j.dp.pool.make_dense_grad_descs, j.dp.pool.grouped_dense_backward, "w x z dy dx dw db work", **size)
    j.dp.sync()
    x, w, b, z = j.rows("x", at), j.t["w"].double().cpu().numpy(), j.t["b"].double().cpu().numpy(), j.rows("z", at)
    want = block.dense_forward(x, w, b, None, block.SILU, True)
    bu.within(z, want["z"], "z")
    bu.within(j.rows("y", at), want["y"], "y")
    want = block.dense_backward(x, w, z, dy, block.SILU)
    bu.within(j.rows("dx", at), want["dx"], "dx", 2)
    bu.within(j.t["dw"].double().cpu().numpy(), want["dw"], "dw", 2)
    bu.within(j.t["db"].double().cpu().numpy(), want["db"], "db")
    assert zero_elsewhere(j.t["dx"], at)
    j.dp.close()


def test_gate_gradients():
    M, K, F, N = (1 << 28) + 40, 8, 8, 8
    made = bu.Buffers(), bu.Buffers(), {}, []
    for name, shape in (("w_in", (K, 2 * F)), ("w_out", (F, N))):
        made[0].add(name, shape, "bf16")
    work = salus.gated_grad_work_bytes(M, F)
    for name, shape, dtype in (("x", (M, K), "bf16"), ("h", (M, F), "bf16"), ("gu", (M, 2 * F), "f32"), ("y", (M, N), "bf16"), ("dy", (M, N), "bf16"), ("dx", (M, K), "bf16"),
                               ("dw_in", (K, 2 * F), "bf16"), ("dw_out", (F, N), "bf16"), ("work", (work,), "raw")):
        made[1].add(name, shape, dtype)
    j = Job(made, dict(w_in=0.35, w_out=0.35, x=1.0))
    spoil(j, work)
    at = seam(M, 1 << 28)
    dy = prepare(j, at, N, 2)
    size = dict(M=M, K=K, F=F, N=N, act=salus.ACT_SILU)
    print("forward", flush=True)
    j.call(j.dp.pool.make_gated_descs, j.dp.pool.grouped_gated_forward, "w_in w_out x h gu y", **size)
    j.dp.sync()
    print("backward", flush=True)
    j.call(j.dp.pool.make_gated_grad_descs, j.dp.pool.grouped_gated_backward, "w_in w_out x h gu dy dx dw_in dw_out work", **size)
    j.dp.sync()
    x, w_in, w_out = j.rows("x", at), j.t["w_in"].double().cpu().numpy(), j.t["w_out"].double().cpu().numpy()
    h, gu = j.rows("h", at), j.rows("gu", at)
    want = block.gated_forward(x, w_in, w_out, None, block.SILU)
    bu.within(gu, want["gu"], "gu")
    bu.within(h, want["h"], "h")
    bu.within(j.rows("y", at), want["y"], "y", 2)
    want = block.gated_backward(x, w_in, w_out, h, gu, dy, block.SILU)
    bu.within(j.rows("dx", at), want["dx"], "dx", 2)
    bu.within(j.t["dw_in"].double().cpu().numpy(), want["dw_in"], "dw_in", 2)
    bu.within(j.t["dw_out"].double().cpu().numpy(), want["dw_out"], "dw_out")
    assert zero_elsewhere(j.t["dx"], at)
    j.dp.close()
