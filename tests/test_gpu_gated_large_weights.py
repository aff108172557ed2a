"""Gated blocks whose two weights are larger than 4 GB each, on the GPU: columns and rows from both ends and from around every 2 GB against the oracle."""
import numpy as np
import pytest
import torch

import block_util as bu
from oracle import block
from paper_1902_04610_amd import salus
from test_gpu_block_large import Job, around

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [3, 40, 200])
def test_gated_with_large_weights(M):
    K, F, N = 32776, 36872, 65544
    made = bu.Buffers(), bu.Buffers(), {}, []
    for name, shape in (("w_in", (K, 2 * F)), ("w_out", (F, N))):
        made[0].add(name, shape, "bf16")
    for name, shape, dtype in (("x", (M, K), "bf16"), ("h", (M, F), "bf16"), ("gu", (M, 2 * F), "f32"), ("y", (M, N), "bf16"), ("dy", (M, N), "bf16"), ("dx", (M, K), "bf16"),
                               ("dw_in", (K, 2 * F), "bf16"), ("dw_out", (F, N), "bf16"), ("work", (salus.gated_grad_work_bytes(M, F),), "raw")):
        made[1].add(name, shape, dtype)
    j = Job(made, dict(w_in=K ** -0.5, w_out=F ** -0.5, x=1.0))
    ns = sorted({0, 1, 127, 128, 20000, N // 2, N - 129, N - 1})
    dy = bu.bf16(np.random.default_rng(M).standard_normal((M, len(ns))))       # all other columns of dY are zero
    j.t["dy"][:, torch.as_tensor(ns, device="cuda")] = torch.from_numpy(dy).to("cuda", torch.bfloat16)
    size = dict(M=M, K=K, F=F, N=N, act=salus.ACT_SILU)
    print("forward", flush=True)
    j.call(j.dp.pool.make_gated_descs, j.dp.pool.grouped_gated_forward, "w_in w_out x h gu y", **size)
    j.dp.sync()
    print("backward", flush=True)
    j.call(j.dp.pool.make_gated_grad_descs, j.dp.pool.grouped_gated_backward, "w_in w_out x h gu dy dx dw_in dw_out work", **size)
    j.dp.sync()
    fs = sorted({0, 1, 63, 64, 9000, F // 2, F - 70, F - 1} | set(around(F, 2 * N)))
    ks = around(K, 4 * F)
    x, h, gu = (j.t[n].double().cpu().numpy() for n in ("x", "h", "gu"))
    # forward: some hidden columns from all of X, some outputs from all of H as it was left
    some = block.gated_forward(x, j.columns("w_in", fs + [F + f for f in fs]), np.zeros((len(fs), 8)), None, block.SILU)
    bu.within(np.concatenate([gu[:, fs], gu[:, [F + f for f in fs]]], 1), some["gu"], "gu")
    bu.within(h[:, fs], some["h"], "h")
    bu.within(j.columns("y", ns), block.rounded(*block.product(h, j.columns("w_out", ns))), "y")
    # backward: rows of dX and of dWin for some of K, rows of dWout for some of F
    want = block.gated_backward(x[:, ks], j.rows("w_in", ks), j.columns("w_out", ns), h, gu, dy, block.SILU)
    bu.within(j.columns("dx", ks), want["dx"], "dx", 2)
    bu.within(j.rows("dw_in", ks), want["dw_in"], "dw_in", 2)
    dw_out = j.rows("dw_out", fs)
    bu.within(dw_out[:, ns], tuple(v[fs] for v in want["dw_out"]), "dw_out")
    assert (np.delete(dw_out, ns, 1) == 0).all()
    j.dp.close()
