"""Rounds of the calls of answering models against the oracle (not a test module)."""
import numpy as np
import torch

from gpu_util import DevicePool
from oracle import answer
from paper_1902_04610_amd import salus, synth

NO_NUMBER = 0x7fc0


def up(v, to=256):
    return (v + to - 1) // to * to


def bf16_bits(a):
    return synth.f32_to_bf16_bits(np.ascontiguousarray(a, np.float32))


def sequences(rng, seqs, page, spare=2, gap=0, tail=0, max_pages=None):
    """seqs: [(new rows, tokens with them)].  Page numbers are drawn without order, unused entries of the table are out of range; `gap` rows in front
    of the first sequence and `tail` behind the last belong to none."""
    need = [-(-max(length, 0) // page) for _, length in seqs]
    n_pages, row = sum(need) + spare, max_pages or max(max(need), 1)
    order = rng.permutation(n_pages)
    table = np.full((len(seqs), row), 0x7fffffff, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :min(n, row)] = order[at:at + min(n, row)]
        at += n
    starts = (gap + np.cumsum([0] + [n for n, _ in seqs])).astype(np.int32)
    return dict(starts=starts, lens=np.array([l for _, l in seqs], np.int32), table=table, n_pages=n_pages, M=max(1, int(starts[-1]) + tail))


class Round:
    """Jobs of one call: each gets a persistent block and a lane, whose buffers are given as arrays; what surrounds them is filled with a pattern and
    looked at again afterwards."""

    def __init__(self, jobs):
        """jobs: [(persistent, lane)], dicts of arrays by name."""
        self.places, total = [], 0
        for persist, lane in jobs:
            sides = []
            for side in (persist, lane):
                at, places = 256, {}
                for name, a in side.items():
                    places[name] = at
                    at += up(max(a.nbytes, 1)) + 256
                sides.append((places, at))
            self.places.append(sides)
            total += sides[0][1] + sides[1][1]
        self.dp = DevicePool(up(total), policy=salus.POLICY_PACK)
        self.dp.buf.fill_(0xa5)
        self.jobs, self.ids, self.off = jobs, [], []
        for (persist, lane), sides in zip(jobs, self.places):
            status, job = self.dp.pool.lane_alloc(sides[0][1], sides[1][1], 0, 0)
            assert status == salus.OK
            self.ids.append(job)
            self.off.append({name + "_off": at for places, _ in sides for name, at in places.items()})
        for j, (persist, lane) in enumerate(jobs):
            for name, a in list(persist.items()) + list(lane.items()):
                self.write(j, name, a)
        self.before = self.dp.buf.clone()

    def address(self, j, name):
        q = self.dp.pool.job_query(self.ids[j])
        return (q.persist_off if name in self.jobs[j][0] else q.lane_off) + self.off[j][name + "_off"]

    def write(self, j, name, a):
        if a.nbytes:
            self.dp.write(self.address(j, name), a)

    def read(self, j, name):
        a = self.jobs[j][0].get(name, self.jobs[j][1].get(name))
        return self.dp.read(self.address(j, name), a.nbytes, a.dtype).reshape(a.shape).copy()

    def check_rest(self, *written):
        """Nothing but the buffers of these names has changed."""
        now, was = self.dp.buf.clone(), self.before.clone()
        for j, (persist, lane) in enumerate(self.jobs):
            for name in written:
                a = persist.get(name, lane.get(name))
                if a is not None:
                    at = self.address(j, name)
                    now[at:at + a.nbytes] = 0
                    was[at:at + a.nbytes] = 0
        assert torch.equal(now, was), "bytes outside the outputs have changed"

    def close(self):
        self.dp.close()


# ---- append ---------------------------------------------------------------------------------------------------------------
def append_job(rng, seqs, Hq, Hkv, D, page, rotary, layout, magnitude=1.0, base=10000.0, **kw):
    q = sequences(rng, seqs, page, **kw)
    M, n_pages = q["M"], q["n_pages"]
    cache = rng.integers(0, 1 << 16, n_pages * Hkv * page * D).astype(np.uint16)
    freq = np.array(salus.rotary_frequencies(rotary, base) if rotary else [], np.float64)
    persist = dict(k=cache, v=cache[::-1].copy(), **(dict(freq=freq) if rotary else {}))
    lane = dict(x=bf16_bits(rng.standard_normal((M, (Hq + 2 * Hkv) * D))), q=np.full((M, Hq * D), NO_NUMBER, np.uint16),
                starts=q["starts"], lens=q["lens"], table=q["table"])
    sizes = dict(M=M, n_seqs=len(seqs), Hq=Hq, Hkv=Hkv, D=D, page=page, n_pages=n_pages, max_pages=q["table"].shape[1], rotary=rotary, layout=layout,
                 magnitude=magnitude)
    return persist, lane, sizes


def append_descs(r, jobs):
    return salus.Pool.make_append_descs(dict(sizes, job=r.ids[j], **r.off[j]) for j, (_, _, sizes) in enumerate(jobs))


def check_append(r, jobs):
    """Rotated elements are off by the roundings of two products and a sum in 32 bits, of their cosine, sine and magnitude (4 * 2^-24 of what they are
    made of), and by their own to bf16, 2^-8; everything else is copied."""
    for j, (persist, lane, sizes) in enumerate(jobs):
        s = {n: v for n, v in sizes.items() if n in ("M", "Hq", "Hkv", "D", "page", "n_pages")}
        q, k, v = answer.append(lane["x"], lane["starts"], lane["lens"], lane["table"], persist.get("freq", []), sizes["layout"],
                                float(np.float32(sizes["magnitude"])), **s)
        got_q, got_k, got_v = r.read(j, "q"), r.read(j, "k").reshape(-1), r.read(j, "v").reshape(-1)
        for row in range(sizes["M"]):
            if row not in q:
                assert (got_q[row] == NO_NUMBER).all(), ("row of no sequence", j, row)
                continue
            want, size = q[row]
            assert (np.abs(answer.bf16_values(got_q[row]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * size).all(), (j, row)
        at = np.array(sorted(k), np.int64)
        rest = np.ones(got_k.size, bool)
        rest[at] = False
        assert np.array_equal(got_k[rest], persist["k"][rest]), ("keys of other places", j)
        if len(at):
            want, size = np.array([k[i] for i in at]).T
            assert (np.abs(answer.bf16_values(got_k[at]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * size).all(), j
        wanted = persist["v"].copy()
        for i, bits in v.items():
            wanted[i] = bits
        assert np.array_equal(got_v, wanted), j


# ---- attention --------------------------------------------------------------------------------------------------------------
def attention_job(rng, seqs, Hq, Hkv, D, page, window=0, scale=None, max_len=None, garbage=True, **kw):
    """Caches whose unused places hold NaNs."""
    q = sequences(rng, seqs, page, **kw)
    M, n_pages = q["M"], q["n_pages"]
    k = np.full(n_pages * Hkv * page * D, NO_NUMBER, np.uint16) if garbage else np.zeros(n_pages * Hkv * page * D, np.uint16)
    v = k.copy()
    d = np.arange(D)
    for s, (_, length) in enumerate(seqs):
        t = np.arange(min(length, page * q["table"].shape[1]))
        p = q["table"][s, t // page].astype(np.int64)[:, None]
        for h in range(Hkv):
            k[answer.key_at(p, h, (t % page)[:, None], d, Hkv, page, D)] = bf16_bits(rng.standard_normal((len(t), D)))
            v[answer.value_at(p, h, (t % page)[:, None], d, Hkv, page, D)] = bf16_bits(rng.standard_normal((len(t), D)))
    limit = max_len or max(1, max(l for _, l in seqs))
    lane = dict(q=bf16_bits(rng.standard_normal((M, Hq * D))), y=np.full((M, Hq * D), NO_NUMBER, np.uint16), starts=q["starts"], lens=q["lens"], table=q["table"])
    work = salus.attention_work_bytes(M, len(seqs), Hq, Hkv, D, limit)
    if work:
        lane["work"] = np.full(work, 0xff, np.uint8)
    sizes = dict(M=M, n_seqs=len(seqs), Hq=Hq, Hkv=Hkv, D=D, page=page, n_pages=n_pages, max_pages=q["table"].shape[1], window=window,
                 scale=D ** -0.5 if scale is None else scale, max_len=limit)
    return dict(k=k, v=v), lane, sizes


def attention_descs(r, jobs):
    return salus.Pool.make_attention_descs(dict(sizes, job=r.ids[j], **r.off[j]) for j, (_, _, sizes) in enumerate(jobs))


def check_attention(r, jobs, beyond=()):
    """An output is off by its own rounding and by that of the weights, 2^-8 of it and of the weighted sizes of the values (A), by the scores' in 32 bits (D products and
    sums of random signs, a few 2^-24 of 10, and an exponent of up to 100: 1e-5 of A each) and the sums' (2^-24 sqrt(n) A): 1e-4 A together.  Rows `beyond` have scores that no float holds: they may hold anything."""
    for j, (persist, lane, sizes) in enumerate(jobs):
        s = {n: v for n, v in sizes.items() if n != "n_seqs" and n != "max_pages"}
        s["scale"] = float(np.float32(s["scale"]))
        want = answer.attention(lane["q"], persist["k"], persist["v"], lane["starts"], lane["lens"], lane["table"], **s)
        got = r.read(j, "y")
        for row in range(sizes["M"]):
            if row not in want:
                assert (got[row] == NO_NUMBER).all(), ("row of no sequence", j, row)
                continue
            if row in beyond:
                continue
            y, size = want[row]
            g = answer.bf16_values(got[row])
            odd = ~np.isfinite(y)
            assert np.array_equal(g[odd], y[odd], equal_nan=True), ("values that are no numbers", j, row, g[odd][:8], y[odd][:8])
            off = np.abs(g - y)[~odd]
            assert (off <= 2.0 ** -8 * (np.abs(y) + size)[~odd] + 1e-4 * size[~odd]).all(), (j, row, off.max(), np.argmax(off))


# ---- sampling ---------------------------------------------------------------------------------------------------------------
def sample_job(logits, params, u, bf16=False, pad=0):
    """logits: M x V floats (of bf16 values if bf16); params: [(temperature, top_k, top_p, min_p)]."""
    M, V = logits.shape
    ld = up(V, 8) + pad
    full = np.full((M, ld), 1e30, np.float32)
    full[:, :V] = logits
    p = np.array([(a, 0, b, c) for a, _, b, c in params], np.float32)
    p.view(np.int32)[:, 1] = [k for _, k, _, _ in params]
    lane = dict(logits=bf16_bits(full) if bf16 else full, params=p, u=np.array(u, np.float32), tokens=np.full(M, -7, np.int32),
                work=np.full(salus.sample_work_bytes(M, V), 0xff, np.uint8))
    return dict(w=np.zeros(64, np.uint8)), lane, dict(M=M, V=V, ld=ld, dtype=salus.BF16 if bf16 else salus.F32)


def sample_descs(r, jobs):
    return salus.Pool.make_sample_descs(dict(sizes, job=r.ids[j], **{n: v for n, v in r.off[j].items() if n != "w_off"}) for j, (_, _, sizes) in enumerate(jobs))


def check_sample(r, jobs):
    for j, (_, lane, sizes) in enumerate(jobs):
        x = answer.bf16_values(lane["logits"]) if sizes["dtype"] == salus.BF16 else lane["logits"]
        p = lane["params"]
        want = [answer.sample(x[i, :sizes["V"]], p[i, 0], int(p.view(np.int32)[i, 1]), float(p[i, 2]), float(p[i, 3]), float(lane["u"][i])) for i in range(sizes["M"])]
        got = r.read(j, "tokens")
        assert got.tolist() == want, (j, [(i, int(g), w, p[i], lane["u"][i]) for i, (g, w) in enumerate(zip(got, want)) if g != w][:4])
