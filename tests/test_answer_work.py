"""A job's largest round of attention leaves room for the sums of all its others (CPU only: launch_recorder.c stands in for the HIP runtime)."""
import json
import os
import random
import re
import subprocess
import sys

import pytest

from paper_1902_04610_amd import build, salus

HERE = os.path.dirname(os.path.abspath(__file__))
HEADS = [(32, 8, 128), (16, 16, 64), (8, 1, 192), (4, 2, 256), (1, 1, 32), (64, 1, 96), (4096, 1, 64)]
# rows, sequences and tokens of the largest round
LARGEST = [(4096, 1, 130000), (64, 64, 130000), (1, 1, 1025), (300, 7, 6000), (100, 100, 1 << 20), (2000, 4, 1100)]

CHILD = r"""
import ctypes, json, sys
from paper_1902_04610_amd import salus as s
take = ctypes.CDLL(None).recorder_take
take.restype = ctypes.c_char_p
up = lambda v: (v + 255) // 256 * 256
out = []
pool = s.Pool(1 << 46, 1 << 45, max_lanes=2, stream=0x50, policy=s.POLICY_PACK)
for (Hq, Hkv, D), (M, S, L), smaller in json.load(sys.stdin):
    pages, cache = -(-L // 32), up(s.cache_bytes(4, Hkv, 32, D))
    at, off = 0, {}
    for name, size in (("q", M * Hq * D * 2), ("y", M * Hq * D * 2), ("starts", 4 * S + 4), ("lens", 4 * S), ("table", 4 * S * pages)):
        off[name + "_off"] = at
        at += up(size)
    work = s.attention_work_bytes(M, S, Hq, Hkv, D, L)
    off["work_off"] = at          # nothing of the lane is behind it
    status, j = pool.lane_alloc(2 * cache, max(256, at + work), 0, 0)
    assert status == s.OK
    for m, n, l, window in smaller:
        descs, keep = pool.make_attention_descs([dict(job=j, M=m, n_seqs=n, Hq=Hq, Hkv=Hkv, D=D, page=32, n_pages=4, max_pages=pages, max_len=l, window=window,
                                                      scale=0.1, k_off=0, v_off=cache, **off)])
        take()
        try:
            rc = pool.grouped_attention(descs, stream=0x50)
        except s.SalusError as e:
            rc = e.code
        out.append([rc, work, s.attention_work_bytes(m, n, Hq, Hkv, D, l), take().decode().splitlines()])
    pool.lane_free(j)
print(json.dumps(out))
"""


def rounds():
    rng = random.Random(3)
    out = []
    for heads in HEADS:
        for M, S, L in LARGEST:
            smaller = [(M, S, L, 0), (1, 1, L, 0), (min(M, 63), 1, L, 0), (min(M, 64), 1, L, 0), (min(M, 2), min(S, 2), L, 0), (min(M, 1528), 1, L, 0)]
            for _ in range(60):
                m, n, l = (max(1, int(round(v ** rng.random()))) for v in (M, S, L))
                smaller.append((rng.choice([m, M]), rng.choice([n, S]), rng.choice([l, L, max(1, L - rng.randrange(400))]), rng.choice([0, 0, 0, 700, 5000])))
            out.append((heads, (M, S, L), smaller))
    return out


def record(folder, asked):
    """[(heads, largest round, call), (status, room of the largest, room of its own, launches)] for each call."""
    if not os.path.exists(build.LIB):
        build.build()
    so = str(folder / "librecorder.so")
    subprocess.check_call(["gcc", "-O1", "-fPIC", "-shared", "-Wall", "-o", so, os.path.join(HERE, "launch_recorder.c")])
    env = dict(os.environ, LD_PRELOAD=":".join(filter(None, [so, os.environ.get("LD_PRELOAD")])), PYTHONPATH=build.ROOT)
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=build.ROOT, env=env, input=json.dumps(asked), stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    each = [(heads, most, call) for heads, most, smaller in asked for call in smaller]
    got = json.loads(r.stdout.splitlines()[-1])
    assert len(got) == len(each)
    return list(zip(each, got))


@pytest.fixture(scope="module")
def outcomes(tmp_path_factory):
    return record(tmp_path_factory.mktemp("recorder"), rounds())


def parts_of(heads, call, line):
    (Hq, Hkv, D), (M, S, L, window) = heads, call
    kernel, grid = re.match(r"launch \S*?(attend_few|attend_many)\S* (\d+) ", line).groups()
    tiles = (M * (Hq // Hkv) // (16 if kernel == "attend_few" else 256 if D <= 128 else 128) + S) * Hkv
    assert int(grid) % tiles == 0
    return int(grid) // tiles


def test_every_smaller_round_has_room_where_the_largest_has(outcomes):
    for (heads, most, call), (rc, work, own, lines) in outcomes:
        assert rc == salus.OK and own <= work, (heads, most, call, rc, work, own)


def test_the_sums_of_the_parts_fit(outcomes):
    several = 0
    for ((Hq, Hkv, D), most, (M, S, L, window)), (rc, work, own, lines) in outcomes:
        parts = parts_of((Hq, Hkv, D), (M, S, L, window), lines[0])
        several += parts > 1
        assert parts == 1 or 4 * M * Hq * parts * (D + 2) <= own, (Hq, Hkv, D, most, M, S, L, window, parts)
    assert several > 200


def test_short_sequences_need_none():
    assert salus.attention_work_bytes(1 << 20, 9, 32, 8, 128, 1024) == 0 < salus.attention_work_bytes(1, 1, 1, 1, 32, 1025)


@pytest.mark.parametrize("heads", HEADS)
def test_room_never_falls_as_a_round_grows(heads):
    sizes = [1, 2, 3, 15, 16, 17, 31, 63, 64, 65, 127, 128, 255, 256, 300, 1000, 1023, 1528, 4000, 9001, 100000]
    lengths = sorted({1, 700, 1024, 1025, 1152, 1153, 1536, 1537, 2000, 4096, 5000, 9000, 16384, 40000, 130000, 131072, 1 << 20, (1 << 30) - 1})
    room = {(M, n, L): salus.attention_work_bytes(M, n, *heads, L) for M in sizes for n in sizes for L in lengths}
    for (M, n, L), bytes_ in room.items():
        for axis, steps in ((0, sizes), (1, sizes), (2, lengths)):
            at = steps.index((M, n, L)[axis])
            if at + 1 < len(steps):
                more = [M, n, L]
                more[axis] = steps[at + 1]
                assert bytes_ <= room[tuple(more)], (M, n, L, more)


# (t tiles; several parts are asked for with at least 512 keys, then evened out and rounded up to 128)
EXACT = [((4, 2, 64), (1, 1, 1024, 0), 1), ((4, 2, 64), (1, 1, 1025, 0), 3),              # t = 2: 3 of 384, two whole and 257 keys
         ((4, 2, 64), (1, 1, 40000, 0), 79),                                              # 79 of 512
         ((2, 1, 64), (3, 1, 3000, 1000), 3), ((2, 1, 64), (3, 1, 3000, 980), 1),         # a span of 1000 + 8 + 32 keys: 3 of 384; of 1020
         ((8, 8, 256), (500, 1, 20000, 4096), 7),                                         # t = 32: 4256 keys by 709 are 7, of 640
         ((8, 8, 256), (500, 1, 20000, 0), 7),                                            # by 3333, of 2944
         ((16, 16, 64), (3000, 1, 3000, 0), 1), ((16, 16, 64), (2800, 1, 3000, 0), 2)]    # t = 192, as many as are wanted; 176: by 2750, 2 of 1536


def test_the_number_of_parts(tmp_path):
    for ((heads, _, call), (rc, _, _, lines)), (_, _, parts) in zip(record(tmp_path, [(heads, call[:3], [call]) for heads, call, _ in EXACT]), EXACT):
        assert rc == salus.OK and parts_of(heads, call, lines[0]) == parts, (heads, call, lines)
