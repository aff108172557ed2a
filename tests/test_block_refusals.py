"""What the transformer-block calls refuse, before anything is launched (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import json
import os
import subprocess
import sys

import pytest

from paper_1902_04610_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))

CHILD = r"""
import ctypes, json, sys
from paper_1902_04610_amd import salus as s
take = ctypes.CDLL(None).recorder_take
take.restype = ctypes.c_char_p
M, K, F, N = 20, 64, 40, 72
up = lambda v: (v + 255) // 256 * 256

def place(sizes):
    at, out = 0, {}
    for name, n in sizes:
        out[name] = at
        at += up(n)
    return out, at

gw, P = place([("w_in_off", K * 2 * F * 2), ("w_out_off", F * N * 2), ("w_off", K * N * 2), ("b_off", N * 2), ("wm_off", 4000), ("wb_off", 2000)])
lane, E = place([("x_off", M * K * 2), ("r_off", M * N * 2), ("y_off", M * N * 4), ("h_off", M * F * 2), ("gu_off", M * 2 * F * 4), ("z_off", M * N * 4),
                 ("dy_off", M * N * 2), ("dx_off", M * K * 2), ("dw_in_off", K * 2 * F * 2), ("dw_out_off", F * N * 2), ("dw_off", K * N * 2),
                 ("db_off", N * 4), ("work_off", s.gated_grad_work_bytes(M, F) + s.dense_grad_work_bytes(M, N)), ("norm_off", 4), ("g_off", 2000)])
off = {**gw, **lane}
pool = s.Pool(1 << 40, up(4 * (P + E)), max_lanes=2, stream=0x50, policy=s.POLICY_PACK)
def job():
    status, j = pool.lane_alloc(P, E, 0, 0)
    assert status == s.OK
    return j
a, b, c = job(), job(), job()      # c shares a lane
lanes = [pool.job_query(j).lane for j in (a, b, c)]
twin = a if lanes[0] == lanes[2] else b
pick = lambda names: {n + "_off": off[n + "_off"] for n in names.split()}
BASE = dict(
    gated=dict(job=a, M=M, K=K, F=F, N=N, act=s.ACT_SILU, **pick("w_in w_out x y h r gu")),
    gated_grad=dict(job=a, M=M, K=K, F=F, N=N, act=s.ACT_SILU, **pick("w_in w_out x h gu dy dx dw_in dw_out work")),
    dense=dict(job=a, M=M, K=K, N=N, act=s.ACT_GELU, y_dtype=s.F32, **pick("w b x y r z")),
    dense_grad=dict(job=a, M=M, K=K, N=N, act=s.ACT_GELU, **pick("w x z dy dx dw db work")),
    clip=dict(job=a, max_norm=1.0, lr=0.1, tensors=[dict(count=1000, dtype=s.BF16, **pick("g wm wb"))], **pick("norm work")),
)
CALLS = dict(gated=(pool.make_gated_descs, pool.grouped_gated_forward), gated_grad=(pool.make_gated_grad_descs, pool.grouped_gated_backward),
             dense=(pool.make_dense_descs, pool.grouped_dense_forward), dense_grad=(pool.make_dense_grad_descs, pool.grouped_dense_backward),
             clip=(pool.make_clip_descs, pool.grouped_clip), clip_sgd=(pool.make_clip_descs, pool.grouped_clip_sgd))

def call(kind, items, n=None):
    make, run = CALLS[kind]
    descs, keep = make(items)
    take()
    try:
        rc = run(descs, n, 0x50)
    except s.SalusError as e:
        rc = e.code
    return [rc, pool.last_error(), take().decode().count("launch")]

def tensor(**change):
    return [dict(BASE["clip"]["tensors"][0], **change)]

out = {}
for kind in CALLS:
    base = BASE["clip" if kind == "clip_sgd" else kind]
    out[kind, "ok"] = call(kind, [base])
    out[kind, "none"] = call(kind, [base], 0)
    out[kind, "two jobs of a lane"] = call(kind, [dict(base, job=twin), dict(base, job=c)])
    out[kind, "two lanes"] = call(kind, [base, dict(base, job=b)])
    out[kind, "no such job"] = call(kind, [dict(base, job=99)])
    changes = {k: v for k, v in base.items() if k.endswith("_off")}
    weights = set(gw)
    for name in changes:
        out[kind, name + " beyond"] = call(kind, [dict(base, **{name: P if name in weights else E})])
        out[kind, name + " far beyond"] = call(kind, [dict(base, **{name: 2 ** 64 - 16})])
        out[kind, name + " misaligned"] = call(kind, [dict(base, **{name: base[name] + 8})])
    if "clip" in kind:
        for what, t in (("count 0", tensor(count=0)), ("count 2^48", tensor(count=1 << 48)), ("dtype", tensor(dtype=2)), ("g beyond", tensor(g_off=E - 16)),
                        ("g misaligned", tensor(g_off=off["g_off"] + 8)), ("twice", tensor() + tensor()), ("g on norm", tensor(g_off=off["norm_off"])), ("no tensors", [])):
            out[kind, what] = call(kind, [dict(base, tensors=t)])
        for v in (0.0, -1.0, float("nan")):
            out[kind, "max_norm %s" % v] = call(kind, [dict(base, max_norm=v)])
        if kind == "clip_sgd":
            out[kind, "wm beyond"] = call(kind, [dict(base, tensors=tensor(wm_off=P - 16))])
            out[kind, "wb absent"] = call(kind, [dict(base, tensors=[{k: v for k, v in tensor()[0].items() if k != "wb_off"}])])
            out[kind, "wb on wm"] = call(kind, [dict(base, tensors=tensor(wb_off=off["wm_off"] + 3984))])
        continue
    for name in [n for n in ("M", "K", "F", "N") if n in base]:
        out[kind, name + " 0"] = call(kind, [dict(base, **{name: 0})])
        out[kind, name + " 2147483648"] = call(kind, [dict(base, **{name: 1 << 31})])
        out[kind, name + " 4294967288"] = call(kind, [dict(base, **{name: 4294967288})])
        if name != "M":
            out[kind, name + " 12"] = call(kind, [dict(base, **{name: 12})])
            out[kind, name + " 2^22"] = call(kind, [dict(base, **{name: 1 << 22})])
    for act in (-1, 4):
        out[kind, "act %d" % act] = call(kind, [dict(base, act=act)])
out["gated", "y on x"] = call("gated", [dict(BASE["gated"], y_off=off["x_off"])])
out["gated", "h in gu"] = call("gated", [dict(BASE["gated"], h_off=off["gu_off"] + 256)])
out["gated", "r is y: ok"] = call("gated", [dict(BASE["gated"], r_off=off["y_off"])])
out["gated", "r is x: ok"] = call("gated", [dict(BASE["gated"], K=N, r_off=off["x_off"], w_in_off=0, gu_off=s.ABSENT, h_off=off["gu_off"])])
out["gated", "r half on y"] = call("gated", [dict(BASE["gated"], r_off=off["y_off"] + 16)])
out["gated_grad", "dx on dy"] = call("gated_grad", [dict(BASE["gated_grad"], dx_off=off["dy_off"])])
out["gated_grad", "work on h"] = call("gated_grad", [dict(BASE["gated_grad"], work_off=off["h_off"])])
out["gated_grad", "no dx: ok"] = call("gated_grad", [dict(BASE["gated_grad"], dx_off=s.ABSENT)])
out["dense", "float y on r"] = call("dense", [dict(BASE["dense"], r_off=off["y_off"])])
out["dense", "bf16 y on r: ok"] = call("dense", [dict(BASE["dense"], y_dtype=s.BF16, r_off=off["y_off"])])
out["dense", "y dtype"] = call("dense", [dict(BASE["dense"], y_dtype=2)])
out["dense_grad", "no z"] = call("dense_grad", [dict(BASE["dense_grad"], z_off=s.ABSENT)])
out["dense_grad", "z without act"] = call("dense_grad", [dict(BASE["dense_grad"], act=s.ACT_NONE)])
out["dense_grad", "neither: ok"] = call("dense_grad", [dict(BASE["dense_grad"], act=s.ACT_NONE, z_off=s.ABSENT, db_off=s.ABSENT, dx_off=s.ABSENT)])
assert pool.switch_out(a) == s.OK
for kind in CALLS:
    out[kind, "evicted"] = call(kind, [BASE["clip" if kind == "clip_sgd" else kind]])
meta = s.Pool(None, 1 << 20)
status, j = meta.lane_alloc(P, E, 0, 0)
for kind, (make, run) in CALLS.items():
    descs, keep = make([dict(BASE["clip" if kind == "clip_sgd" else kind], job=j)])
    out[kind, "no memory"] = [getattr(meta, run.__name__)(descs), meta.last_error(), 0]
    out[kind, "null"] = [getattr(s.lib(), "salus_" + run.__name__)(pool._h, None, 1, None), pool.last_error(), 0]
    out[kind, "no pool"] = [getattr(s.lib(), "salus_" + run.__name__)(None, descs, 1, None), "", 0]
print(json.dumps([[list(k), v] for k, v in out.items()]))
"""


@pytest.fixture(scope="module")
def outcomes(tmp_path_factory):
    if not os.path.exists(build.LIB):
        build.build()
    so = str(tmp_path_factory.mktemp("recorder") / "librecorder.so")
    subprocess.check_call(["gcc", "-O1", "-fPIC", "-shared", "-Wall", "-o", so, os.path.join(HERE, "launch_recorder.c")])
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, [so, os.environ.get("LD_PRELOAD")])), PYTHONPATH=build.ROOT)
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=build.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return {tuple(k): v for k, v in json.loads(r.stdout.splitlines()[-1])}


SPECIAL = {"ok": 0, "none": 0, "two lanes": 0, "two jobs of a lane": -4, "evicted": -3}


def test_every_case_has_the_expected_status(outcomes):
    assert len(outcomes) > 150
    wrong = {k: v for k, v in outcomes.items()
             if v[0] != (0 if k[1].endswith(": ok") else SPECIAL.get(k[1], -1)) or (v[0] != 0 and (v[2] != 0 or (not v[1] and k[1] != "no pool")))}
    assert not wrong, wrong


def test_what_is_accepted_is_launched(outcomes):
    for k, v in outcomes.items():
        if v[0] == 0:
            assert (v[2] > 0) == (k[1] != "none"), (k, v)


def test_messages_name_the_fault(outcomes):
    assert "persistent" in outcomes["gated", "w_in_off beyond"][1]
    assert "lane" in outcomes["gated", "x_off far beyond"][1]
    assert "overlap" in outcomes["gated", "h in gu"][1]
    assert "multiples of 8" in outcomes["dense", "K 12"][1]
    assert "2^31" in outcomes["dense_grad", "M 2147483648"][1] and "2^31" in outcomes["gated", "M 4294967288"][1]
    assert "activation" in outcomes["dense_grad", "act 4"][1]
    assert "max_norm" in outcomes["clip", "max_norm nan"][1]
    assert "resident" in outcomes["clip_sgd", "evicted"][1]
