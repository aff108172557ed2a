"""Which attention kernels a call takes, and in how many parts (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import json
import os
import re
import subprocess
import sys

import pytest

from paper_1902_04610_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))

# new rows, sequences, Hq, Hkv, D, max_len, window
CASES = [
    (1, 1, 4, 2, 64, 1024, 0), (1, 1, 4, 2, 64, 1025, 0), (1, 1, 4, 2, 64, 40000, 0), (1, 1, 4, 2, 64, 40000, 700), (63, 1, 1, 1, 64, 300, 0), (64, 1, 1, 1, 64, 300, 0),
    (63, 1, 2, 2, 128, 4000, 0), (16, 1, 8, 2, 192, 4000, 0), (31, 2, 4, 1, 64, 300, 0), (32, 2, 4, 1, 64, 300, 0), (3000, 3000, 1, 1, 32, 9000, 0), (3000, 1, 16, 16, 64, 3000, 0),
    (500, 1, 8, 8, 256, 20000, 4096), (500, 1, 8, 8, 256, 20000, (1 << 32) - 1), (1, 1, 1, 1, 32, (1 << 30) - 1, 0), (200, 1, 1, 1, 32, (1 << 30) - 1, 5000),
]

CHILD = r"""
import ctypes, json, sys
from paper_1902_04610_amd import salus as s
take = ctypes.CDLL(None).recorder_take
take.restype = ctypes.c_char_p
out = []
pool = s.Pool(1 << 46, 1 << 44, max_lanes=2, stream=0x50, policy=s.POLICY_PACK)
up = lambda v: (v + 255) // 256 * 256
for M, S, Hq, Hkv, D, max_len, window in json.loads(sys.argv[1]):
    max_pages = -(-max_len // 32)
    cache, work = up(s.cache_bytes(4, Hkv, 32, D)), s.attention_work_bytes(M, S, Hq, Hkv, D, max_len)
    at, off = 0, {}
    for name, size in (("q", M * Hq * D * 2), ("y", M * Hq * D * 2), ("starts", 4 * S + 4), ("lens", 4 * S), ("table", 4 * S * max_pages), ("work", work)):
        off[name + "_off"] = at
        at += up(size)
    status, j = pool.lane_alloc(2 * cache, up(at) + 256, 0, 0)
    assert status == s.OK
    descs, keep = pool.make_attention_descs([dict(job=j, M=M, n_seqs=S, Hq=Hq, Hkv=Hkv, D=D, page=32, n_pages=4, max_pages=max_pages, max_len=max_len, window=window,
                                                  scale=0.1, k_off=0, v_off=cache, **off)])
    take()
    assert pool.grouped_attention(descs, stream=0x50) == s.OK, pool.last_error()
    out.append([work, take().decode().splitlines()])
    pool.lane_free(j)
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if not os.path.exists(build.LIB):
        build.build()
    so = str(tmp_path_factory.mktemp("recorder") / "librecorder.so")
    subprocess.check_call(["gcc", "-O1", "-fPIC", "-shared", "-Wall", "-o", so, os.path.join(HERE, "launch_recorder.c")])
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, [so, os.environ.get("LD_PRELOAD")])), PYTHONPATH=build.ROOT)
    r = subprocess.run([sys.executable, "-c", CHILD, json.dumps(CASES)], cwd=build.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    out = []
    for work, lines in json.loads(r.stdout.splitlines()[-1]):
        found = [re.match(r"launch \S*?(attend_few|attend_many|join_parts)\S* (\d+) (\d+) \S+$", line).groups() for line in lines]
        out.append((work, [(name, int(grid)) for name, grid, _ in found]))
    return out


@pytest.mark.parametrize("number", range(len(CASES)))
def test_the_kernel_its_grid_and_the_room_for_parts(launches, number):
    M, S, Hq, Hkv, D, max_len, window = CASES[number]
    work, found = launches[number]
    G = Hq // Hkv
    many = M * G >= 64 * S
    columns = 16 if not many else 256 if D <= 128 else 128
    tiles = (M * G // columns + S) * Hkv
    name, grid = found[0]
    assert name == ("attend_many" if many else "attend_few")
    assert grid % tiles == 0
    parts = grid // tiles
    # a part has at least 512 keys once there is more than one; what there is room for is what the longest unwindowed call leaves
    keys = min(max_len, window + columns // G + 32) if window else max_len
    assert parts == 1 if keys <= 1024 else parts <= -(-keys // 512)
    assert (len(found) == 2 and found[1][0] == "join_parts") == (parts > 1)
    assert parts == 1 or 4 * M * Hq * parts * (D + 2) <= work
    if max_len <= 1024:
        assert work == 0
    if parts > 1:
        assert found[1][1] == tiles * (columns if parts > 16 else columns // 16)


def test_few_tiles_of_long_sequences_have_many_parts(launches):
    grids = [found[0][1] for _, found in launches]
    assert grids[2] == 2 * 79 and grids[14] > 400 and grids[3] == 2
