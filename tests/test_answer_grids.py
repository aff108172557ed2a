"""Grids of the kernels of answering models for the largest rounds (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import json
import os
import re
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
up = lambda v: (v + 255) // 256 * 256
kind, jobs, sizes = json.loads(sys.argv[1])

def place(buffers):
    at, off = 0, {}
    for name, size in buffers:
        off[name + "_off"] = at
        at += up(size)
    return off, at

if kind == "sample":
    M, V = sizes["M"], sizes["V"]
    off, E = place([("logits", M * sizes["ld"] * 2), ("params", 16 * M), ("u", 4 * M), ("tokens", 4 * M), ("work", s.sample_work_bytes(M, V))])
    off, P, sizes = dict(off), 256, dict(sizes, dtype=s.BF16)
else:
    M, n, row, Hq, Hkv, D = (sizes[k] for k in ("M", "n_seqs", "max_pages", "Hq", "Hkv", "D"))
    held, P = place([("k", s.cache_bytes(sizes["n_pages"], Hkv, sizes["page"], D)), ("v", s.cache_bytes(sizes["n_pages"], Hkv, sizes["page"], D))])
    rows = [("q", M * Hq * D * 2), ("x", M * (Hq + 2 * Hkv) * D * 2)] if kind == "append" else [("q", M * Hq * D * 2), ("y", M * Hq * D * 2)]
    off, E = place(rows + [("starts", 4 * n + 4), ("lens", 4 * n), ("table", 4 * n * row)])
    off = {**held, **off}
    if kind == "append":
        sizes = dict(sizes, rotary=0, layout=0, magnitude=1.0, freq_off=s.ABSENT)
    else:
        sizes = dict(dict(window=0, scale=0.1, work_off=0), **sizes)
pool = s.Pool(1 << 50, up(jobs * (P + E)), max_lanes=jobs, stream=0x50, policy=s.POLICY_PACK)
ids = []
for _ in range(jobs):
    status, j = pool.lane_alloc(P, E, 0, 0)
    assert status == s.OK
    ids.append(j)
make, run = dict(sample=(pool.make_sample_descs, pool.grouped_sample), append=(pool.make_append_descs, pool.grouped_append),
                 attention=(pool.make_attention_descs, pool.grouped_attention))[kind]
descs, keep = make([dict(sizes, job=j, **off) for j in ids])
take()
try:
    rc = run(descs, stream=0x50)
except s.SalusError as e:
    rc = e.code
print(json.dumps([rc, pool.last_error(), take().decode().splitlines()]))
"""


def call(so_dir, kind, jobs, sizes):
    """Status, message, what was launched."""
    if not os.path.exists(build.LIB):
        build.build()
    so = str(so_dir / "librecorder.so")
    subprocess.check_call(["gcc", "-O1", "-fPIC", "-shared", "-Wall", "-o", so, os.path.join(HERE, "launch_recorder.c")])
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, [so, os.environ.get("LD_PRELOAD")])), PYTHONPATH=build.ROOT)
    r = subprocess.run([sys.executable, "-c", CHILD, json.dumps([kind, jobs, sizes])], cwd=build.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.splitlines()[-1])


def launches(so_dir, kind, jobs, sizes):
    rc, error, lines = call(so_dir, kind, jobs, sizes)
    assert rc == 0, (rc, error)
    return [(name, int(grid), int(block)) for name, grid, block in
            (re.match(r"launch \S*?(attend_few|attend_many|join_parts|append_rows|slice_rows|choose_rows)\S* (\d+) (\d+) \S+$", line).groups() for line in lines)]


def check(found, name, workgroups):
    mine = [(grid, block) for n, grid, block in found if n == name]
    assert sum(grid for grid, _ in mine) == workgroups, (name, mine)
    assert all(grid * block < 1 << 32 for grid, block in mine), (name, mine)


# (of a pool that 288 GB hold)
@pytest.mark.parametrize("M,V", [(1 << 22, 8), ((1 << 22) + 5, 1), (1 << 19, 128256)])
def test_rows_of_logits(M, V, tmp_path):
    found = launches(tmp_path, "sample", 1, dict(M=M, V=V, ld=(V + 7) // 8 * 8))
    check(found, "slice_rows", M * -(-V // 8192))
    check(found, "choose_rows", M)


CACHED = dict(page=32, n_pages=4, max_pages=1, max_len=32)


def test_many_columns(tmp_path):
    M, n, H = 1 << 25, 1 << 19, 32
    check(launches(tmp_path, "attention", 1, dict(CACHED, M=M, n_seqs=n, Hq=H, Hkv=H, D=32)), "attend_many", (M // 256 + n) * H)


def test_few_columns_and_appends_of_millions_of_sequences(tmp_path):
    n = 60_000_000
    check(launches(tmp_path, "attention", 1, dict(CACHED, M=n, n_seqs=n, Hq=1, Hkv=1, D=32)), "attend_few", n // 16 + n)
    sizes = {k: v for k, v in CACHED.items() if k != "max_len"}
    check(launches(tmp_path, "append", 1, dict(sizes, M=n, n_seqs=n, Hq=1, Hkv=1, D=32)), "append_rows", n // 8 + 2 * n)


def test_jobs_whose_workgroups_no_launch_numbers_together(tmp_path):
    n, jobs = 60_000_000, 30
    sizes = {k: v for k, v in CACHED.items() if k != "max_len"}
    check(launches(tmp_path, "append", jobs, dict(sizes, M=1, n_seqs=n, Hq=1, Hkv=1, D=32)), "append_rows", jobs * 2 * n)
