"""Rounds of transformer-block operators on a device pool, for the GPU tests (not a test module).

All of the pool's memory that no call may touch, and everything that is to be written, holds NaNs before the call; afterwards
what lies outside the written buffers has to be as it was, to the byte."""
import numpy as np

from gpu_util import DevicePool
from oracle import block
from paper_1902_04610_amd import salus, synth

ESZ = {"bf16": 2, "f32": 4, "f64": 8, "raw": 1}


def bf16(a):
    """Values that bf16 holds, as float64."""
    return synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(np.asarray(a, np.float32))).astype(np.float64)


def to_bytes(a, dtype):
    a = np.asarray(a)
    if dtype == "bf16":
        return synth.f32_to_bf16_bits(a.astype(np.float32)).reshape(-1).view(np.uint8)
    return np.ascontiguousarray(a.astype(np.float32)).reshape(-1).view(np.uint8)


def up(v, to=16):
    return (v + to - 1) // to * to


class Buffers:
    """name -> (offset, shape, dtype) in one region; `pad` bytes after each."""

    def __init__(self, pad=0):
        self.at, self.end, self.pad = {}, 0, pad

    def add(self, name, shape, dtype):
        n = int(np.prod(shape)) * ESZ[dtype]
        self.at[name] = (self.end, tuple(shape), dtype)
        self.end += up(n) + self.pad


class Round:
    """jobs: list of (persistent Buffers, lane Buffers, {name: values}, names that the call writes)."""

    def __init__(self, jobs, pad_jobs=0, stream=None):
        sizes = [(up(max(p.end, 16), 256), up(max(l.end, 16), 256)) for p, l, _, _ in jobs]
        self.dp = DevicePool(sum(p + e for p, e in sizes) + 4096, policy=salus.POLICY_PACK)
        self.jobs, self.ids = jobs, []
        image = np.full(self.dp.capacity // 2, 0x7fc1, np.uint16).view(np.uint8)      # a NaN as bf16, and as float
        self.base = []
        for (p, l, data, _), (P, E) in zip(jobs, sizes):
            status, job = self.dp.pool.lane_alloc(P, E, 0, 0)
            assert status == salus.OK
            self.ids.append(job)
        for (p, l, data, _), job in zip(jobs, self.ids):
            q = self.dp.pool.job_query(job)
            self.base.append({**{n: (q.persist_off + o, s, t) for n, (o, s, t) in p.at.items()},
                              **{n: (q.lane_off + o, s, t) for n, (o, s, t) in l.at.items()}})
            for name, v in data.items():
                off, shape, t = self.base[-1][name]
                b = to_bytes(v, t)
                assert b.size == int(np.prod(shape)) * ESZ[t], name
                image[off:off + b.size] = b
        self.image = image
        self.restore()

    def restore(self):
        self.dp.write(0, self.image)
        self.dp.sync()

    def load(self, i, name, v):
        """New values for an input, in the image as well."""
        off, shape, t = self.base[i][name]
        b = to_bytes(v, t)
        self.image[off:off + b.size] = b
        self.dp.write(off, b)

    def offsets(self, i, names):
        p, l = self.jobs[i][0], self.jobs[i][1]
        return {n + "_off": (p.at[n] if n in p.at else l.at[n])[0] for n in names.split() if n in p.at or n in l.at}

    def read(self, i, name):
        off, shape, t = self.base[i][name]
        n = int(np.prod(shape))
        raw = self.dp.read(off, n * ESZ[t])
        if t == "bf16":
            return synth.bf16_bits_to_f32(raw.view(np.uint16)).astype(np.float64).reshape(shape)
        return raw.view(np.float32).astype(np.float64).reshape(shape)

    def untouched(self):
        """Nothing but the written buffers has changed."""
        now = self.dp.read(0, self.dp.capacity)
        same = now == self.image
        for (_, _, _, written), base in zip(self.jobs, self.base):
            for name in written:
                off, shape, t = base[name]
                same[off:off + int(np.prod(shape)) * ESZ[t]] = True
        assert same.all(), np.flatnonzero(~same)[:8]

    def close(self):
        self.dp.close()


def within(got, expected, what, roundings=1):
    """Every value inside its bound, and all of them together no further off than as many roundings to bf16 as there are."""
    v, e = expected
    bad = ~(np.abs(got - v) <= e + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], v[bad][:4], np.broadcast_to(e, v.shape)[bad][:4])
    if roundings:
        size = np.sqrt((v * v).sum())
        assert np.sqrt(((got - v) ** 2).sum()) <= (np.sqrt(roundings) * block.HALF + 1e-4) * size + 1e-30, what


def gated_job(rng, M, K, F, N, act=block.SILU, residual=True, train=False, in_place=False, scale=1.0, pad=0):
    p, l = Buffers(pad), Buffers(pad)
    p.add("w_in", (K, 2 * F), "bf16")
    p.add("w_out", (F, N), "bf16")
    l.add("x", (M, K), "bf16")
    if residual and not in_place:
        l.add("r", (M, N), "bf16")
    l.add("y", (M, N), "bf16")
    l.add("h", (M, F), "bf16")
    d = dict(w_in=bf16(rng.standard_normal((K, 2 * F)) / np.sqrt(K)), w_out=bf16(rng.standard_normal((F, N)) / np.sqrt(F)),
             x=bf16(rng.standard_normal((M, K)) * scale))
    if residual:
        d["y" if in_place else "r"] = bf16(rng.standard_normal((M, N)))
    written = ["y", "h"]
    if train:
        l.add("gu", (M, 2 * F), "f32")
        l.add("dy", (M, N), "bf16")
        l.add("dx", (M, K), "bf16")
        l.add("dw_in", (K, 2 * F), "bf16")
        l.add("dw_out", (F, N), "bf16")
        l.add("work", (salus.gated_grad_work_bytes(M, F),), "raw")
        d["dy"] = bf16(rng.standard_normal((M, N)) / M)
        written += ["gu", "dx", "dw_in", "dw_out", "work"]
    size = dict(M=M, K=K, F=F, N=N, act=act)
    return dict(size=size, residual=residual, in_place=in_place, train=train, parts=(p, l, d, written))


def gated_descs(rnd, jobs):
    items = []
    for i, j in enumerate(jobs):
        it = dict(j["size"], job=rnd.ids[i], **rnd.offsets(i, "w_in w_out x y h r gu"))
        if j["in_place"]:
            it["r_off"] = it["y_off"]
        items.append(it)
    return salus.Pool.make_gated_descs(items)


def gated_grad_descs(rnd, jobs, dx=True):
    return salus.Pool.make_gated_grad_descs(dict(j["size"], job=rnd.ids[i], **rnd.offsets(
        i, "w_in w_out x h gu dy dw_in dw_out work" + (" dx" if dx else ""))) for i, j in enumerate(jobs))


def run_gated(jobs, stream=None):
    rnd = Round([j["parts"] for j in jobs])
    stream = rnd.dp.stream if stream is None else stream
    descs, keep = gated_descs(rnd, jobs)
    assert rnd.dp.pool.grouped_gated_forward(descs, stream=stream) == salus.OK, rnd.dp.pool.last_error()
    train = [j["train"] for j in jobs]
    assert len(set(train)) == 1
    if train[0]:
        grads, keep = gated_grad_descs(rnd, jobs)
        assert rnd.dp.pool.grouped_gated_backward(grads, stream=stream) == salus.OK, rnd.dp.pool.last_error()
    rnd.dp.sync()
    return rnd


def check_gated(rnd, jobs):
    rnd.untouched()
    for i, j in enumerate(jobs):
        d, s = j["parts"][2], j["size"]
        r = d.get("y" if j["in_place"] else "r")
        what = (i, s)
        want = block.gated_forward(d["x"], d["w_in"], d["w_out"], r, s["act"])
        h = rnd.read(i, "h")
        within(h, want["h"], what + ("h",))
        within(rnd.read(i, "y"), want["y"], what + ("y",), 2)
        if not j["train"]:
            continue
        gu = rnd.read(i, "gu")
        within(gu, want["gu"], what + ("gu",))
        want = block.gated_backward(d["x"], d["w_in"], d["w_out"], h, gu, d["dy"], s["act"])
        within(rnd.read(i, "dx"), want["dx"], what + ("dx",), 2)
        within(rnd.read(i, "dw_in"), want["dw_in"], what + ("dw_in",), 2)
        within(rnd.read(i, "dw_out"), want["dw_out"], what + ("dw_out",))


def dense_job(rng, M, K, N, act=block.GELU, out="bf16", bias=True, residual=True, train=False, in_place=False, pad=0):
    p, l = Buffers(pad), Buffers(pad)
    p.add("w", (K, N), "bf16")
    d = dict(w=bf16(rng.standard_normal((K, N)) / np.sqrt(K)), x=bf16(rng.standard_normal((M, K))))
    if bias:
        p.add("b", (N,), "bf16")
        d["b"] = bf16(rng.standard_normal(N) * 0.5)
    l.add("x", (M, K), "bf16")
    if residual and not in_place:
        l.add("r", (M, N), "bf16")
    l.add("y", (M, N), out)
    if residual:
        d["y" if in_place else "r"] = bf16(rng.standard_normal((M, N)))
    written = ["y"]
    if train:
        if act != block.NONE:
            l.add("z", (M, N), "f32")
            written.append("z")
        l.add("dy", (M, N), "bf16")
        l.add("dx", (M, K), "bf16")
        l.add("dw", (K, N), "bf16")
        if bias:
            l.add("db", (N,), "f32")
            written.append("db")
        l.add("work", (salus.dense_grad_work_bytes(M, N),), "raw")
        d["dy"] = bf16(rng.standard_normal((M, N)) / M)
        written += ["dx", "dw", "work"]
    return dict(size=dict(M=M, K=K, N=N, act=act), out=out, residual=residual, in_place=in_place, train=train, parts=(p, l, d, written))


def dense_descs(rnd, jobs):
    items = []
    for i, j in enumerate(jobs):
        it = dict(j["size"], job=rnd.ids[i], y_dtype=salus.F32 if j["out"] == "f32" else salus.BF16, **rnd.offsets(i, "w b x y r z"))
        if j["in_place"]:
            it["r_off"] = it["y_off"]
        items.append(it)
    return salus.Pool.make_dense_descs(items)


def dense_grad_descs(rnd, jobs):
    return salus.Pool.make_dense_grad_descs(dict(j["size"], job=rnd.ids[i], **rnd.offsets(i, "w x z dy dx dw db work")) for i, j in enumerate(jobs))


def run_dense(jobs, stream=None):
    rnd = Round([j["parts"] for j in jobs])
    stream = rnd.dp.stream if stream is None else stream
    descs, keep = dense_descs(rnd, jobs)
    assert rnd.dp.pool.grouped_dense_forward(descs, stream=stream) == salus.OK, rnd.dp.pool.last_error()
    if jobs[0]["train"]:
        grads, keep = dense_grad_descs(rnd, jobs)
        assert rnd.dp.pool.grouped_dense_backward(grads, stream=stream) == salus.OK, rnd.dp.pool.last_error()
    rnd.dp.sync()
    return rnd


def check_dense(rnd, jobs):
    rnd.untouched()
    for i, j in enumerate(jobs):
        d, s = j["parts"][2], j["size"]
        what = (i, s, j["out"])
        want = block.dense_forward(d["x"], d["w"], d.get("b"), d.get("y" if j["in_place"] else "r"), s["act"], j["out"] == "bf16")
        within(rnd.read(i, "y"), want["y"], what + ("y",))
        if not j["train"]:
            continue
        z = None
        if s["act"] != block.NONE:
            z = rnd.read(i, "z")
            within(z, want["z"], what + ("z",))
        want = block.dense_backward(d["x"], d["w"], z, d["dy"], s["act"])
        within(rnd.read(i, "dx"), want["dx"], what + ("dx",), 2)
        within(rnd.read(i, "dw"), want["dw"], what + ("dw",), 2)
        if "b" in d:
            within(rnd.read(i, "db"), want["db"], what + ("db",))


def clip_job(rng, counts, dtypes, max_norm=1.0, lr=0.05, scale=1.0, sgd=False):
    p, l, d, written = Buffers(), Buffers(), {}, ["norm", "work"]
    total = sum(counts)
    for t, (n, dt) in enumerate(zip(counts, dtypes)):
        l.add(f"g{t}", (n,), dt)
        g = rng.standard_normal(n) * scale / np.sqrt(total)
        d[f"g{t}"] = bf16(g) if dt == "bf16" else g.astype(np.float32).astype(np.float64)
        if sgd:
            p.add(f"wm{t}", (n,), "f32")
            p.add(f"wb{t}", (n,), "bf16")
            d[f"wm{t}"] = rng.standard_normal(n).astype(np.float32).astype(np.float64)
            written += [f"wm{t}", f"wb{t}"]
        else:
            written.append(f"g{t}")
    l.add("norm", (1,), "f32")
    l.add("work", (salus.clip_work_bytes([dict(g_off=0, count=n, dtype=0) for n in counts]),), "raw")
    return dict(counts=counts, dtypes=dtypes, max_norm=max_norm, lr=lr, sgd=sgd, parts=(p, l, d, written))


def clip_descs(rnd, jobs):
    items = []
    for i, j in enumerate(jobs):
        tensors = []
        for t, (n, dt) in enumerate(zip(j["counts"], j["dtypes"])):
            o = rnd.offsets(i, f"g{t} wm{t} wb{t}")
            tensors.append({"count": n, "dtype": salus.BF16 if dt == "bf16" else salus.F32,
                            **{k.replace(str(t), ""): v for k, v in o.items()}})
        items.append(dict(job=rnd.ids[i], tensors=tensors, max_norm=j["max_norm"], lr=j["lr"], **rnd.offsets(i, "norm work")))
    return salus.Pool.make_clip_descs(items)


def run_clip(jobs, stream=None):
    rnd = Round([j["parts"] for j in jobs])
    descs, keep = clip_descs(rnd, jobs)
    call = rnd.dp.pool.grouped_clip_sgd if jobs[0]["sgd"] else rnd.dp.pool.grouped_clip
    assert call(descs, stream=rnd.dp.stream if stream is None else stream) == salus.OK, rnd.dp.pool.last_error()
    rnd.dp.sync()
    return rnd


def check_clip(rnd, jobs):
    rnd.untouched()
    for i, j in enumerate(jobs):
        d = j["parts"][2]
        g = [d[f"g{t}"] for t in range(len(j["counts"]))]
        norm, c = block.clip(g, np.float64(np.float32(j["max_norm"])))
        got = rnd.read(i, "norm")[0]
        assert abs(got - norm) <= 2 * block.STEP * norm, (i, got, norm)
        lr = np.float64(np.float32(j["lr"]))
        for t, (v, dt) in enumerate(zip(g, j["dtypes"])):
            scaled = c * v
            es = 3 * block.STEP * np.abs(scaled)             # the coefficient, the product
            if not j["sgd"]:
                bound = np.zeros_like(v) if c == 1 else es + (block.HALF if dt == "bf16" else 0) * (np.abs(scaled) + es)
                within(rnd.read(i, f"g{t}"), (scaled, bound), (i, t, "g"), 0)
                continue
            want = d[f"wm{t}"] - lr * scaled
            e = lr * (es + block.STEP * np.abs(scaled)) + block.STEP * np.abs(want) * (1 + 1e-6)
            wm = rnd.read(i, f"wm{t}")
            within(wm, (want, e), (i, t, "wm"), 0)
            assert np.array_equal(rnd.read(i, f"wb{t}"), bf16(wm)), (i, t, "wb")
