"""What packed language-model jobs do between their dense layers when they answer, as cases that can be timed and compared.

Every case is one packed call over the jobs of a round, each in a lane of its own of one pool over one device buffer.  Kinds:

  append    queries and keys of new tokens rotated by their positions, keys and values stored in the pages of each job's cache
  attend    attention of the new tokens' queries over the cache: single tokens, prompts, chunks of prompts
  sample    one token from each row of logits: temperature, top-k, top-p, min-p, a given random number

`run` computes the operators in elementary torch operations in 32 bits (angles of positions, and sums of a vocabulary's weights, in
64), rounded once at the end; with `own` it makes the library's calls on the same buffers.  A case holds plain values; lengths
and numbers of sequences are drawn from the case's own `mix` number, so that `work` knows them, and the data come from the seed of
`prepare`.

Where a cache keeps element d of token t of page p and head h (D elements a head, `page` tokens a page), in elements from its beginning:
  keys     (p Hkv + h) page D + ((t / 32) (D / 8) + d / 8) 256 + (t % 32) 8 + d % 8
  values   (p Hkv + h) page D + ((t / 8) D + d) 8 + t % 8
"""
import math

import numpy as np
import torch

own = False


# ---- cases ------------------------------------------------------------------------------------------------------------
def _attend(jobs, seqs, rows, past, Hq, Hkv, D, page, window=0, mix=1):
    return dict(kind="attend", jobs=jobs, seqs=seqs, rows=rows, past=past, Hq=Hq, Hkv=Hkv, D=D, page=page, window=window, mix=mix)


def _append(jobs, seqs, rows, past, Hq, Hkv, D, page, rotary, layout, factor=1.0, mix=1):
    return dict(kind="append", jobs=jobs, seqs=seqs, rows=rows, past=past, Hq=Hq, Hkv=Hkv, D=D, page=page, rotary=rotary,
                layout=layout, factor=factor, mix=mix)


def _sample(jobs, rows, V, dtype, flat=False, mix=1):
    return dict(kind="sample", jobs=jobs, rows=rows, V=V, dtype=dtype, flat=flat, mix=mix)


def listed():
    return [
        # one token of one sequence, a short conversation: latency
        dict(_attend(1, "1", "1", "700", 16, 4, 64, 32), name="attend_one_token"),
        # a decoding round of 16 resident models, 1 - 16 sequences each, conversations of all lengths
        dict(_attend(16, "1..16", "1", "1..6000", 32, 8, 128, 64, mix=5), name="attend_packed_decode"),
        # few sequences with long documents behind them
        dict(_attend(2, "2", "1", "100000..130000", 32, 8, 128, 256, mix=3), name="attend_long_context"),
        # prompts of four models, compute bound
        dict(_attend(4, "3", "1000..5000", "0", 32, 8, 128, 64, mix=2), name="attend_prompts"),
        # chunks of long prompts behind what is cached, a window of keys, a key head for every query head
        dict(_attend(2, "2", "512", "8000..20000", 16, 16, 64, 128, window=4096, mix=4), name="attend_chunks_window"),
        # one token of one sequence: latency
        dict(_append(1, "1", "1", "700", 16, 4, 64, 32, 64, "half"), name="append_one_token"),
        # the decoding round's
        dict(_append(16, "1..16", "1", "1..6000", 32, 8, 128, 64, 128, "half", mix=5), name="append_packed_decode"),
        # prompts, part of each head rotated, frequencies scaled for long contexts
        dict(_append(4, "3", "500..5000", "0..100", 32, 8, 128, 64, 64, "interleaved", 4.0, mix=2), name="append_prompts"),
        # one row of logits: latency
        dict(_sample(1, "1", 32000, "f32"), name="sample_one_row"),
        # the decoding round's rows, an odd vocabulary
        dict(_sample(16, "1..16", 50257, "f32", mix=5), name="sample_packed_decode"),
        # many rows of one model with a large vocabulary
        dict(_sample(1, "256", 128256, "bf16"), name="sample_large"),
    ]


def _logint(rng, lo, hi, mult=1):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random() / mult)) * mult))


def _span(rng, lo, hi, most):
    """A range of sizes as text, its ends drawn."""
    a = _logint(rng, lo, hi)
    return "%d..%d" % (a, _logint(rng, a, max(a, min(hi, most * a))))


def draw(rng):
    """Sizes over the ranges of the listed cases; never more work than the largest of its kind."""
    kind, mix = rng.choice(["attend", "attend", "attend", "append", "append", "sample", "sample"]), rng.randrange(1 << 20)
    if kind == "sample":
        V = _logint(rng, 1000, 200000)
        rows = _span(rng, 1, 64, 8)
        jobs = max(1, min(_logint(rng, 1, 32), int(30e6 // (V * int(rows.split("..")[1])))))
        return _sample(jobs, rows, V, rng.choice(["f32", "bf16"]), rng.random() < 0.2, mix)
    D, Hkv = rng.choice([32, 64, 64, 96, 128, 128, 128, 192, 256]), rng.choice([1, 2, 4, 8, 16])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 7, 8])
    page = rng.choice([32, 64, 128, 256])
    if kind == "append":
        rows = "1" if rng.random() < 0.5 else _span(rng, 2, 4000, 8)
        seqs = _span(rng, 1, 16, 8)
        most = int(rows.split("..")[-1]) * int(seqs.split("..")[-1]) * (Hq + 2 * Hkv) * D
        rotary = 2 * rng.randint(1, D // 2) if rng.random() < 0.4 else D
        return _append(max(1, min(_logint(rng, 1, 24), int(1.5e8 // most))), seqs, rows, _span(rng, 1, 30000, 8), Hq, Hkv, D, page, rotary,
                       rng.choice(["half", "half", "interleaved"]), rng.choice([1.0, 1.0, 8.0]), mix)
    window = 0 if rng.random() < 0.7 else _logint(rng, 16, 8000)
    if rng.random() < 0.6:              # single tokens, now and then a few proposed ones
        rows, past = rng.choice(["1", "1", "1", "2..5"]), _span(rng, 1, 60000, 30)
        seqs = _span(rng, 1, 24, 8)
        each = int(seqs.split("..")[-1]) * int(past.split("..")[-1]) * Hkv * D * 4
        if each > 1.5e9:
            seqs, each = "1..2", 2 * int(past.split("..")[-1]) * Hkv * D * 4
        return _attend(max(1, min(_logint(rng, 1, 24), int(1.5e9 // each))), seqs, rows, past, Hq, Hkv, D, page, window, mix)
    rows, past = _span(rng, 6, 2500, 6), _span(rng, 1, 8000, 30) if rng.random() < 0.5 else "0"
    n, m = int(rows.split("..")[-1]), int(past.split("..")[-1])
    each = n * (n / 2 + m) * Hq * D * 4
    seqs = "1" if each > 5e10 else _span(rng, 1, 4, 4)
    return _attend(max(1, min(_logint(rng, 1, 8), int(3e11 // (each * int(seqs.split("..")[-1]))))), seqs, rows, past, Hq, Hkv, D, page, window, mix)


# ---- sizes and places ---------------------------------------------------------------------------------------------------
def _pick(spec, r):
    if ".." not in spec:
        return int(spec)
    lo, hi = (int(v) for v in spec.split(".."))
    return int(round(lo * (hi / lo) ** r.random_sample())) if lo else r.randint(lo, hi + 1)


def _lengths(case):
    """For each job the (new tokens, tokens with the new ones) of its sequences; rows of logits for sampling."""
    r, out = np.random.RandomState(case["mix"]), []
    for _ in range(case["jobs"]):
        if case["kind"] == "sample":
            out.append(_pick(case["rows"], r))
        else:
            job = []
            for _ in range(_pick(case["seqs"], r)):
                n = _pick(case["rows"], r)
                job.append((n, n + _pick(case["past"], r)))
            out.append(job)
    return out


def _up(v, to=256):
    return (v + to - 1) // to * to


B16, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
_SIZE = {B16: 2, F32: 4, F64: 8, I32: 4, U8: 1}


def _pages(case, job):
    """Pages of a job's cache (some to spare) and the entries of a row of its page table."""
    each = [_up(length, case["page"]) // case["page"] for _, length in job]
    return sum(each) + 3, max(each)


def _ld(V):
    return _up(V, 8)


def _buffers(case, job):
    """(name, shape, type) of a job's buffers: those that stay with the job, and those of its lane."""
    if case["kind"] == "sample":
        t = B16 if case["dtype"] == "bf16" else F32
        return [("w", (64,), B16)], [("logits", (job, _ld(case["V"])), t), ("params", (job, 4), F32), ("u", (job,), F32), ("tokens", (job,), I32)]
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    n_pages, row = _pages(case, job)
    M = sum(n for n, _ in job)
    cache = (n_pages * Hkv * case["page"] * D,)
    stay = [("k", cache, B16), ("v", cache, B16)]
    lane = [("q", (M, Hq * D), B16), ("starts", (len(job) + 1,), I32), ("lens", (len(job),), I32), ("table", (len(job), row), I32)]
    if case["kind"] == "append":
        return stay + [("freq", (max(1, case["rotary"] // 2),), F64)], lane + [("x", (M, (Hq + 2 * Hkv) * D), B16)]
    return stay, lane + [("y", (M, Hq * D), B16)]


def _place(bufs):
    at, places = 0, []
    for name, shape, t in bufs:
        places.append((name, shape, t, at))
        at += _up(int(np.prod(shape)) * _SIZE[t])
    return places, at


BASE, TRAINED = 10000.0, 4096


def _frequencies(case):
    """Radians a token for every pair; with a factor, pairs that turn less than once in the trained length are slowed by it, those that turn more
    than 32 times are not, with a ramp between."""
    R = case["rotary"]
    f = BASE ** (-np.arange(0, R, 2, dtype=np.float64) / R)
    keep = np.clip((TRAINED * f / (2 * np.pi) - 1) / (32 - 1), 0, 1)
    return f * keep + f / case["factor"] * (1 - keep)


def _magnitude(case):
    return float(np.float32(0.1 * math.log(case["factor"]) + 1))


def _job_data(case, job, g):
    """One job's inputs, by name of the buffer; everything else is written by the calls."""
    def normal(shape, scale=1.0, t=B16):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(t)
    if case["kind"] == "sample":
        def uniform(lo=0.0, hi=1.0):
            return lo + (hi - lo) * torch.rand(job, generator=g, device="cuda")
        V, t = case["V"], B16 if case["dtype"] == "bf16" else F32
        logits = normal((job, _ld(V)), 2.0, F32)
        if not case["flat"]:            # some forty tokens take nearly all of the weight, as a trained model's do
            at = torch.randint(V, (job, 40), generator=g, device="cuda")
            logits.scatter_add_(1, at, 6 + 8 * torch.rand(job, 40, generator=g, device="cuda"))
        logits[:, V:] = float("-inf")
        kind = uniform()
        temperature = torch.where(kind < 0.06, torch.zeros_like(kind), uniform(0.6, 1.2))
        top_k = torch.where((kind > 0.3) & (kind < 0.7), uniform(5, 200).floor(), torch.zeros_like(kind)).to(I32)
        top_p = torch.where((kind > 0.5) & (kind < 0.9), uniform(0.8, 0.98), torch.ones_like(kind))
        min_p = torch.where(kind > 0.8, uniform(0.02, 0.1), torch.zeros_like(kind))
        params = torch.stack([temperature, top_k.view(F32), top_p, min_p], 1)
        return dict(logits=logits.to(t), params=params, u=uniform(2.0 ** -20, 1 - 2.0 ** -20))
    n_pages, row = _pages(case, job)
    cache = (n_pages * case["Hkv"] * case["page"] * case["D"],)
    M = sum(n for n, _ in job)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(I32)
    table, at = torch.full((len(job), row), -1, dtype=I32, device="cuda"), 0
    for s, (_, length) in enumerate(job):
        count = _up(length, case["page"]) // case["page"]
        table[s, :count] = order[at:at + count]
        at += count
    d = dict(k=normal(cache), v=normal(cache), table=table,
             starts=torch.tensor(np.cumsum([0] + [n for n, _ in job]), dtype=I32, device="cuda"),
             lens=torch.tensor([length for _, length in job], dtype=I32, device="cuda"))
    if case["kind"] == "append":
        return dict(d, x=normal((M, (case["Hq"] + 2 * case["Hkv"]) * case["D"])), freq=torch.from_numpy(_frequencies(case)).cuda())
    return dict(d, q=normal((M, case["Hq"] * case["D"])))


class _Job:
    pass


class _State:
    """One device buffer with every job's buffers in it; with the library, the pool over it and the call's descriptors."""

    def __init__(self, case, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.case, self.kind, self.jobs, self.pool = case, case["kind"], [], None
        jobs = _lengths(case)
        plan = []
        for job in jobs:
            stay, lane = _buffers(case, job)
            if own:
                work = self.work_bytes(job)
                lane = lane + ([("work", (work,), U8)] if work else [])
            plan.append((_place(stay), _place(lane)))
        self.capacity = sum(p + e for (_, p), (_, e) in plan)
        self.buf = torch.zeros(self.capacity, dtype=U8, device="cuda")
        low, high = 0, self.capacity
        for job, ((stay, p), (lane, e)) in zip(jobs, plan):
            high -= e                    # persistent blocks grow up from 0, lanes down from the end
            j = _Job()
            j.job, j.P, j.E, j.low, j.high, j.off = job, p, e, low, high, {}
            for places, base in ((stay, low), (lane, high)):
                for name, shape, t, at in places:
                    n = int(np.prod(shape)) * _SIZE[t]
                    setattr(j, name, self.buf[base + at:base + at + n].view(t).view(*shape))
                    j.off[name] = at
            for name, v in _job_data(case, job, g).items():
                getattr(j, name).copy_(v)
            low += p
            self.jobs.append(j)
        if own:
            self.attach()

    def work_bytes(self, job):
        from paper_1902_04610_amd import salus
        case = self.case
        if self.kind == "sample":
            return salus.sample_work_bytes(job, case["V"])
        if self.kind == "append":
            return 0
        return salus.attention_work_bytes(sum(n for n, _ in job), len(job), case["Hq"], case["Hkv"], case["D"], max(length for _, length in job))

    def attach(self):
        from paper_1902_04610_amd import salus
        self.stream = torch.cuda.current_stream().cuda_stream
        self.pool = salus.Pool(self.buf.data_ptr(), self.capacity, policy=salus.POLICY_PACK, stream=self.stream)
        case, items = self.case, []
        for j in self.jobs:
            status, j.id = self.pool.lane_alloc(j.P, j.E, 0, 0)
            q = self.pool.job_query(j.id)
            assert status == salus.OK and q.persist_off == j.low and q.lane_off == j.high, self.pool.last_error()
            off = {name + "_off": at for name, at in j.off.items() if name != "w"}
            if self.kind == "sample":
                items.append(dict(job=j.id, M=j.job, V=case["V"], ld=_ld(case["V"]), dtype=salus.BF16 if case["dtype"] == "bf16" else salus.F32, **off))
                continue
            n_pages, row = _pages(case, j.job)
            item = dict(job=j.id, M=j.q.shape[0], n_seqs=len(j.job), Hq=case["Hq"], Hkv=case["Hkv"], D=case["D"], page=case["page"],
                        n_pages=n_pages, max_pages=row, **off)
            if self.kind == "append":
                item.update(rotary=case["rotary"], layout=salus.ROTARY_HALF if case["layout"] == "half" else salus.ROTARY_INTERLEAVED,
                            magnitude=_magnitude(case))
            else:
                item.update(max_len=max(length for _, length in j.job), window=case["window"], scale=case["D"] ** -0.5)
            items.append(item)
        make = dict(append=salus.Pool.make_append_descs, attend=salus.Pool.make_attention_descs, sample=salus.Pool.make_sample_descs)[self.kind]
        self.call = make(items)

    def __del__(self):
        if self.pool is not None:
            torch.cuda.synchronize()
            self.pool.close()


def prepare(case, seed):
    return _State(case, seed)


# ---- one pass -------------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        p = s.pool
        call = dict(append=p.grouped_append, attend=p.grouped_attention, sample=p.grouped_sample)[s.kind]
        assert call(s.call[0], len(s.jobs), s.stream) == 0, p.last_error()
        return [_outputs(s.kind, j) for j in s.jobs]
    return [_PLAIN[s.kind](s.case, j) for j in s.jobs]


def _outputs(kind, j):
    return dict(append=lambda: [j.q, j.k, j.v], attend=lambda: [j.y], sample=lambda: [j.tokens])[kind]()


def _slots(case, table, t):
    """Element of the caches at which tokens t of one sequence begin: of their keys' first element, of their values'; Hkv x tokens."""
    page, D = case["page"], case["D"]
    block = (table[t // page].long() * case["Hkv"] + torch.arange(case["Hkv"], device="cuda")[:, None]) * page * D
    i = t % page
    return block + i // 32 * (32 * D) + i % 32 * 8, block + i // 8 * (8 * D) + i % 8


def _steps(case):
    """The same for the elements of a head: what is added for element d of the keys, of the values."""
    d = torch.arange(case["D"], device="cuda")
    return d // 8 * 256 + d % 8, d * 8


def _plain_append(case, j):
    Hq, Hkv, D, R = case["Hq"], case["Hkv"], case["D"], case["rotary"]
    at = 0
    j.q.zero_()
    for s, (n, length) in enumerate(j.job):
        p = torch.arange(length - n, length, device="cuda")
        x = j.x[at:at + n].float().view(n, Hq + 2 * Hkv, D)
        angle = p.double()[:, None] * j.freq[None]
        c, si = (torch.cos(angle) * _magnitude(case)).float()[:, None], (torch.sin(angle) * _magnitude(case)).float()[:, None]
        turned = x[:, :Hq + Hkv].clone()
        first, second = (slice(0, R // 2), slice(R // 2, R)) if case["layout"] == "half" else (slice(0, R, 2), slice(1, R, 2))
        a, b = x[:, :Hq + Hkv, first], x[:, :Hq + Hkv, second]
        turned[:, :, first] = a * c - b * si
        turned[:, :, second] = a * si + b * c
        j.q[at:at + n] = turned[:, :Hq].reshape(n, Hq * D).to(B16)
        k_at, v_at = _slots(case, j.table[s], p)
        k_step, v_step = _steps(case)
        j.k[k_at[:, :, None] + k_step] = turned[:, Hq:].transpose(0, 1).to(B16)
        j.v[v_at[:, :, None] + v_step] = x[:, Hq + Hkv:].transpose(0, 1).to(B16)
        at += n
    return [j.q, j.k, j.v]


def _plain_attend(case, j):
    Hq, Hkv, D, window = case["Hq"], case["Hkv"], case["D"], case["window"]
    at = 0
    for s, (n, length) in enumerate(j.job):
        t = torch.arange(length, device="cuda")
        k_at, v_at = _slots(case, j.table[s], t)
        k_step, v_step = _steps(case)
        p = torch.arange(length - n, length, device="cuda")[:, None]
        hidden = t[None] > p
        if window:
            hidden |= t[None] <= p - window
        for h in range(Hkv):
            k, v = j.k[k_at[h, :, None] + k_step].float(), j.v[v_at[h, :, None] + v_step].float()
            G = Hq // Hkv
            cols = slice(h * G * D, (h + 1) * G * D)
            q = j.q[at:at + n, cols].float().view(n, G, D).transpose(0, 1).reshape(G * n, D)
            score = (q @ k.t() * D ** -0.5).view(G, n, length).masked_fill_(hidden, float("-inf"))
            w = torch.exp(score - score.amax(2, keepdim=True))
            w /= w.sum(2, keepdim=True)
            j.y[at:at + n, cols] = (w.view(G * n, length) @ v).view(G, n, D).transpose(0, 1).reshape(n, G * D).to(B16)
        at += n
    return [j.y]


def _plain_sample(case, j):
    V = case["V"]
    T, k, p, m = j.params[:, 0].double(), j.params[:, 1].contiguous().view(I32), j.params[:, 2].double(), j.params[:, 3].double()
    logits, order = torch.sort(j.logits[:, :V].double(), dim=1, descending=True, stable=True)
    w = torch.exp((logits - logits[:, :1]) / torch.where(T > 0, T, torch.ones_like(T))[:, None])
    place = torch.arange(V, device="cuda")[None]
    w *= (place < torch.where(k > 0, k, torch.full_like(k, V))[:, None])
    before = torch.cumsum(w, 1) - w
    kept = (before < p[:, None] * w.sum(1, keepdim=True)) & (w >= m[:, None]) | (place == 0)
    w *= kept
    weight = torch.zeros_like(w).scatter_(1, order, w)
    run_sum = torch.cumsum(weight, 1)
    token = (run_sum <= j.u.double()[:, None] * weight.sum(1, keepdim=True)).sum(1)
    j.tokens.copy_(torch.where(T > 0, token, order[:, 0]))
    return [j.tokens]


_PLAIN = dict(append=_plain_append, attend=_plain_attend, sample=_plain_sample)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def _seen(n, length, window):
    """(query row, key) pairs of one sequence, and the keys that any row sees."""
    p = np.arange(length - n, length, dtype=np.float64)
    first = np.maximum(p - window + 1, 0) if window else np.zeros_like(p)
    return float((p + 1 - first).sum()), float(length - first[0])


def work(case):
    jobs = _lengths(case)
    if case["kind"] == "sample":
        rows = sum(jobs)
        return {"bytes": rows * (case["V"] * (2 if case["dtype"] == "bf16" else 4) + 24), "flops": 4 * rows * case["V"]}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    M = sum(n for job in jobs for n, _ in job)
    if case["kind"] == "append":
        return {"bytes": 2 * M * (Hq + 2 * Hkv) * D * 2, "flops": 3 * M * (Hq + Hkv) * case["rotary"]}
    pairs = keys = 0
    for job in jobs:
        for n, length in job:
            a, b = _seen(n, length, case["window"])
            pairs, keys = pairs + a, keys + b
    return {"bytes": keys * Hkv * D * 4 + 2 * M * Hq * D * 2, "flops": 4 * pairs * Hq * D}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------
def exact(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    define = dict(append=_exact_append, attend=_exact_attend, sample=_exact_sample)[case["kind"]]
    return [define(case, job, _job_data(case, job, g)) for job in _lengths(case)]


def _unpacked(case, cache, values):
    """A cache's elements as pages x heads x tokens x elements (a view)."""
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    if values:
        return cache.view(-1, Hkv, page // 8, D, 8).permute(0, 1, 2, 4, 3)       # pages, heads, tokens / 8, tokens % 8, elements
    return cache.view(-1, Hkv, page // 32, D // 8, 32, 8).permute(0, 1, 2, 4, 3, 5)


def _exact_append(case, job, d):
    Hq, Hkv, D, R, page = case["Hq"], case["Hkv"], case["D"], case["rotary"], case["page"]
    q_out, k, v = [], d["k"].double(), d["v"].double()
    k_view, v_view = _unpacked(case, k, False), _unpacked(case, v, True)
    rows = torch.split(d["x"].double(), [n for n, _ in job])
    for s, (n, length) in enumerate(job):
        t = torch.arange(length - n, length, device="cuda")
        q, key, val = (part.unflatten(1, (-1, D)) for part in torch.split(rows[s], [Hq * D, Hkv * D, Hkv * D], 1))
        turn = torch.polar(torch.full((n, 1), _magnitude(case), dtype=F64, device="cuda"), t[:, None] * d["freq"])[:, None]

        def rotate(h):
            head, rest = h[..., :R], h[..., R:]
            if case["layout"] == "half":
                z = torch.view_as_real(torch.complex(*head.chunk(2, -1)) * turn).transpose(-1, -2).flatten(-2)
            else:
                z = torch.view_as_real(torch.view_as_complex(head.unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
            return torch.cat([z, rest], -1)
        q_out.append(rotate(q).flatten(1))
        where = d["table"][s].long()[t // page]
        i = t % page
        k_view[where, :, i // 32, i % 32] = rotate(key).unflatten(-1, (-1, 8))
        v_view[where, :, i // 8, i % 8] = val
    return [torch.cat(q_out), k, v]


def _exact_attend(case, job, d):
    Hq, Hkv, D, page, window = case["Hq"], case["Hkv"], case["D"], case["page"], case["window"]
    k_view, v_view = _unpacked(case, d["k"], False), _unpacked(case, d["v"], True)
    out = []
    for s, q in enumerate(torch.split(d["q"], [n for n, _ in job])):
        n, length = job[s]
        pages = d["table"][s, :_up(length, page) // page].long()
        k = k_view[pages].flatten(4).flatten(2, 3).transpose(0, 1).flatten(1, 2)[:, :length]       # heads x tokens x elements
        v = v_view[pages].flatten(2, 3).transpose(0, 1).flatten(1, 2)[:, :length]
        key = torch.arange(length, device="cuda")
        head = q.unflatten(1, (Hkv, Hq // Hkv, D))
        blocks = []
        for r in range(0, n, 512):
            at = torch.arange(length - n + r, length - n + min(n, r + 512), device="cuda")
            sees = (key <= at[:, None]) & (key > at[:, None] - window if window else key >= 0)
            heads = []
            for h in range(Hkv):
                kh, vh = k[h].double(), v[h].double()
                for e in range(Hq // Hkv):
                    logit = (head[r:r + 512, h, e].double() @ kh.mT) / math.sqrt(D)
                    heads.append(torch.softmax(logit.where(sees, torch.full_like(logit, -torch.inf)), -1) @ vh)
            blocks.append(torch.cat(heads, 1))
        out.append(torch.cat(blocks))
    return [torch.cat(out)]


def _exact_sample(case, job, d):
    V, tokens = case["V"], []
    table = d["logits"][:, :V].double().cpu().numpy()
    params, u = d["params"].cpu().numpy(), d["u"].cpu().numpy().astype(np.float64)
    for row, (T, _, p, m), k, r in zip(table, params.astype(np.float64), params[:, 1].copy().view(np.int32), u):
        if T <= 0:
            tokens.append(int(np.argmax(row)))
            continue
        weight = np.exp((row - row.max()) / T)
        order = np.argsort(-row, kind="stable")
        if k > 0:
            order = order[:k]
        total = np.cumsum(weight[order])
        order = order[:1 + int(np.searchsorted(total, p * total[-1], side="left"))]
        order = np.sort(order[weight[order] >= m])
        total = np.cumsum(weight[order])
        tokens.append(int(order[np.searchsorted(total, r * total[-1], side="right")]))
    return [torch.tensor(tokens, dtype=I32, device="cuda")]
