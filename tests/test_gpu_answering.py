"""The calls of answering models as they are used: one after the other, recorded and replayed, on several streams, on caches and rows behind 4 GiB, on
keys in parts."""
import numpy as np
import pytest
import torch

from answer_util import (NO_NUMBER, Round, append_descs, append_job, attention_descs, attention_job, bf16_bits, check_append, check_attention, check_sample,
                         sample_descs, sample_job, sequences, up)
from gpu_util import DevicePool
from oracle import answer
from paper_1902_04610_amd import salus

pytestmark = pytest.mark.gpu
HALF = salus.ROTARY_HALF


# ---- keys in parts ------------------------------------------------------------------------------------------------------------
def attend(jobs):
    r = Round([(p, l) for p, l, _ in jobs])
    descs, keep = attention_descs(r, jobs)
    assert r.dp.pool.grouped_attention(descs, stream=r.dp.stream) == salus.OK, r.dp.pool.last_error()
    r.dp.sync()
    check_attention(r, jobs)
    r.check_rest("y", "work")
    r.close()


@pytest.mark.parametrize("limit", [1025, 6000, 30000])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 192, 256])
def test_parts_of_all_widths(D, limit):
    """Single tokens, a few and a prompt; lengths around the ends of parts of 512."""
    rng = np.random.default_rng(D + limit)
    for seqs in ([(1, 1025)], [(1, 512), (1, 513), (2, 511), (1, 0), (3, 1024), (1, 1)], [(90, 1024), (30, 30)]):
        attend([attention_job(rng, seqs, 3, 1, D, 64, max_len=limit, max_pages=-(-limit // 64), gap=1)])


@pytest.mark.parametrize("rows", [2, 80])
@pytest.mark.parametrize("limit", [1100, 20000])
def test_parts_with_values_and_keys_that_are_no_numbers(limit, rows):
    """Whatever part they are in, they reach those who see them."""
    for which, bits in (("v", 0x7f80), ("v", 0x7fc0), ("k", 0x7f80), ("k", 0x7fc0)):
        p, l, sizes = attention_job(np.random.default_rng(rows), [(rows, 1090)], 2, 1, 64, 32, max_len=limit, max_pages=-(-limit // 32))
        for token in (1089, 1089 - rows // 2, 40):
            if token == 40 and which == "k":
                continue
            at = int(l["table"][0, token // 32]), 0, token % 32
            p[which][answer.value_at(*at, 9, 1, 32, 64) if which == "v" else answer.key_at(*at, np.arange(64), 1, 32, 64)] = bits
        attend([(p, l, sizes)])


def test_parts_whose_pages_are_not_there():
    p, l, sizes = attention_job(np.random.default_rng(3), [(1, 1400), (2, 1300)], 2, 1, 64, 32, max_len=9000, max_pages=282)
    l["table"][0, 16:32] = -1          # the second part of the first sequence
    l["table"][1, :] = 1 << 30         # all of the second
    attend([(p, l, sizes)])


# ---- together -----------------------------------------------------------------------------------------------------------------
class Answering:
    """Jobs that answer: a dense layer to queries, keys and values, the cache, attention, a dense layer to logits, a token; M rows for any of their steps."""

    def __init__(self, rng, shapes, M, limit):
        self.M, self.E, self.V, self.seqs, jobs, self.sizes = M, [], [], [], [], []
        for H, Hq, Hkv, D, page, V, n in shapes:
            N, q = (Hq + 2 * Hkv) * D, sequences(rng, [(0, limit)] * n, page)
            cache = np.full(q["n_pages"] * Hkv * page * D, NO_NUMBER, np.uint16)
            persist = dict(k=cache, v=cache.copy(), freq=np.array(salus.rotary_frequencies(D), np.float64), w_in=bf16_bits(rng.standard_normal((H, N)) * H ** -0.5),
                           w_out=bf16_bits(rng.standard_normal((Hq * D, V)) * 3 * (Hq * D) ** -0.5))
            lane = dict(h=np.zeros((M, H), np.uint16), x=np.zeros((M, N), np.uint16), q=np.zeros((M, Hq * D), np.uint16), y=np.zeros((M, Hq * D), np.uint16),
                        logits=np.zeros((M, V), np.float32), params=np.zeros((M, 4), np.float32), u=np.zeros(M, np.float32), tokens=np.zeros(M, np.int32),
                        starts=np.zeros(n + 1, np.int32), lens=np.zeros(n, np.int32), table=q["table"],
                        awork=np.zeros(max(256, salus.attention_work_bytes(M, n, Hq, Hkv, D, limit)), np.uint8),
                        swork=np.zeros(salus.sample_work_bytes(M, V), np.uint8))
            jobs.append((persist, lane))
            self.sizes.append(dict(M=M, n_seqs=n, Hq=Hq, Hkv=Hkv, D=D, page=page, n_pages=q["n_pages"], max_pages=q["table"].shape[1]))
            self.E.append(bf16_bits(rng.standard_normal((V, H))))
            self.V.append(V)
            self.seqs.append([[] for _ in range(n)])      # tokens so far
        self.r, self.limit = Round(jobs), limit
        r, P = self.r, salus.Pool
        off = lambda j, *names, **as_: dict({n + "_off": r.off[j][n + "_off"] for n in names}, **{n: r.off[j][v + "_off"] for n, v in as_.items()})
        both = list(enumerate(self.sizes))
        dense = lambda j, K, N, w, x, y, dtype: dict(job=r.ids[j], M=M, K=K, N=N, act=salus.ACT_NONE, y_dtype=dtype, b_off=salus.ABSENT, r_off=salus.ABSENT,
                                                     z_off=salus.ABSENT, **off(j, w_off=w, x_off=x, y_off=y))
        self.append_sizes = [dict(s, rotary=s["D"], layout=HALF, magnitude=1.0) for s in self.sizes]
        self.attention_sizes = [dict(s, window=0, scale=s["D"] ** -0.5, max_len=limit) for s in self.sizes]
        self.sample_sizes = [dict(M=M, V=V, ld=V, dtype=salus.F32) for V in self.V]
        self.calls = [
            (r.dp.pool.grouped_dense_forward, P.make_dense_descs([dense(j, self.E[j].shape[1], (s["Hq"] + 2 * s["Hkv"]) * s["D"], "w_in", "h", "x", salus.BF16) for j, s in both])),
            (r.dp.pool.grouped_append, P.make_append_descs([dict(s, job=r.ids[j], **off(j, "x", "q", "k", "v", "freq", "starts", "lens", "table"))
                                                            for j, s in enumerate(self.append_sizes)])),
            (r.dp.pool.grouped_attention, P.make_attention_descs([dict(s, job=r.ids[j], **off(j, "q", "y", "k", "v", "starts", "lens", "table", work_off="awork"))
                                                                  for j, s in enumerate(self.attention_sizes)])),
            (r.dp.pool.grouped_dense_forward, P.make_dense_descs([dense(j, s["Hq"] * s["D"], self.V[j], "w_out", "y", "logits", salus.F32) for j, s in both])),
            (r.dp.pool.grouped_sample, P.make_sample_descs([dict(s, job=r.ids[j], **off(j, "logits", "params", "u", "tokens", work_off="swork"))
                                                            for j, s in enumerate(self.sample_sizes)])),
        ]

    def call(self, stream):
        for f, made in self.calls:
            assert f(made[0], stream=stream) == salus.OK, self.r.dp.pool.last_error()

    def load(self, rng, new):
        """new[j][s]: tokens that sequence s of job j goes on with."""
        r = self.r
        for j, seqs in enumerate(self.seqs):
            for s, tokens in enumerate(new[j]):
                seqs[s] += tokens
            starts = np.cumsum([0] + [len(t) for t in new[j]]).astype(np.int32)
            rows = np.zeros_like(r.jobs[j][1]["h"])
            rows[:starts[-1]] = self.E[j][[t for tokens in new[j] for t in tokens]]
            params = np.zeros((self.M, 4), np.float32)
            params[:, 0], params[:, 2] = rng.choice([0.0, 0.8, 1.3], self.M), rng.choice([0.7, 1.0], self.M)
            params.view(np.int32)[:, 1] = rng.choice([0, 5, 40], self.M)
            for name, a in dict(h=rows, starts=starts, lens=np.array([len(t) for t in seqs], np.int32), params=params, u=rng.random(self.M).astype(np.float32)).items():
                r.write(j, name, a)
            for name in ("q", "y"):
                r.write(j, name, np.full(r.jobs[j][1][name].shape, NO_NUMBER, np.uint16))

    def outputs(self):
        return [self.r.read(j, name) for j in range(len(self.V)) for name in ("x", "q", "k", "v", "y", "logits", "tokens")]

    def check(self, before):
        """Each call by the oracle, from what the one before it has left."""
        r = self.r
        now = [{name: r.read(j, name) for name in ("x", "q", "y", "k", "v", "freq", "logits", "params", "u", "starts", "lens", "table")} for j in range(len(self.V))]
        check_append(r, [(dict(n, k=b[0], v=b[1]), n, s) for n, b, s in zip(now, before, self.append_sizes)])
        check_attention(r, [(n, n, s) for n, s in zip(now, self.attention_sizes)])
        check_sample(r, [(n, n, s) for n, s in zip(now, self.sample_sizes)])

    def last_tokens(self):
        out = []
        for j in range(len(self.V)):
            starts, tokens = self.r.read(j, "starts"), self.r.read(j, "tokens")
            out.append([[int(tokens[e - 1])] if e > b else [] for b, e in zip(starts[:-1], starts[1:])])
        return out


SHAPES = [(64, 4, 2, 64, 32, 1000, 3), (96, 8, 1, 128, 64, 5008, 2), (40, 2, 2, 32, 32, 264, 1)]


def steps(rng, model, turns):
    """Prompts, then token by token; now and then a sequence waits or takes several."""
    new = [[[int(t) for t in rng.integers(0, V, 3 + 2 * s)] for s in range(len(seqs))] for V, seqs in zip(model.V, model.seqs)]
    for turn in range(turns):
        yield new
        new = model.last_tokens()
        if turn % 3 == 1:
            new[0][0] = []
        if turn % 3 == 2:
            new[1][1] = new[1][1] * 4


def test_prompts_and_tokens_one_after_the_other():
    rng = np.random.default_rng(1)
    model = Answering(rng, SHAPES, 16, 200)
    for new in steps(rng, model, 7):
        model.load(rng, new)
        before = [(model.r.read(j, "k"), model.r.read(j, "v")) for j in range(3)]
        model.call(model.r.dp.stream)
        model.r.dp.sync()
        model.check(before)
    model.r.close()


def test_a_recorded_step_replays_with_new_lengths_rows_and_parameters():
    """Room for 2000 tokens a sequence, so keys in parts; between the replays the same step eagerly."""
    rng = np.random.default_rng(2)
    model = Answering(rng, SHAPES, 16, 2000)
    r = model.r
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        model.call(side.cuda_stream)
    for turn, new in enumerate(steps(rng, model, 6)):
        model.load(rng, new)
        before, state, results = [(r.read(j, "k"), r.read(j, "v")) for j in range(3)], r.dp.buf.clone(), []
        for replay in (False, True):
            r.dp.buf.copy_(state)
            torch.cuda.synchronize()
            graph.replay() if replay else model.call(r.dp.stream)
            torch.cuda.synchronize()
            results.append(model.outputs())
        assert all(np.array_equal(a, b, equal_nan=a.dtype == np.float32) for a, b in zip(*results)), turn
        model.check(before)
    r.close()


def test_two_graphs_that_share_everything():
    """Two recordings of the same step, one after the other on the same workspaces: each replay gives the eager step's results."""
    rng = np.random.default_rng(5)
    model = Answering(rng, SHAPES[:1], 8, 1500)
    r, graphs = model.r, []
    for _ in range(2):
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            model.call(side.cuda_stream)
        graphs.append(graph)
    model.load(rng, [[[1, 2], [3], [4, 5, 6]]])
    state = r.dp.buf.clone()
    model.call(r.dp.stream)
    r.dp.sync()
    want = model.outputs()
    for turn in range(4):
        r.dp.buf.copy_(state)
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(a, b, equal_nan=a.dtype == np.float32) for a, b in zip(model.outputs(), want)), turn      # rows of no sequence have NaN as logits
    r.close()


def test_streams_other_than_the_current_one():
    """Two jobs on streams of their own, nothing between them; the calls' results are those of the current stream's."""
    rng = np.random.default_rng(4)
    appends = [append_job(rng, [(40, 400), (1, 90)], 4, 2, 64, 32, 64, HALF) for _ in range(2)]
    attends = [attention_job(rng, [(3, 1700), (1, 90)], 4, 2, 64, 32) for _ in range(2)]
    samples = [sample_job((rng.standard_normal((4, 20000)) * 2).astype(np.float32), [(1.0, 50, 0.9, 0.0), (0.7, 0, 0.8, 0.0), (1.0, 0, 1.0, 0.01), (0.0, 0, 1.0, 0.0)],
                          rng.random(4)) for _ in range(2)]
    for jobs, make, call, check in ((appends, append_descs, "grouped_append", check_append), (attends, attention_descs, "grouped_attention", check_attention),
                                    (samples, sample_descs, "grouped_sample", check_sample)):
        r = Round([(p, l) for p, l, _ in jobs])
        descs, keep = make(r, jobs)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in jobs]
        for j, stream in enumerate(streams):
            one = type(descs[j]) * 1
            assert getattr(r.dp.pool, call)(one(descs[j]), n=1, stream=stream.cuda_stream) == salus.OK, r.dp.pool.last_error()
        for stream in streams:
            stream.synchronize()
        check(r, jobs)
        r.close()


# ---- behind 4 GiB -----------------------------------------------------------------------------------------------------------------
class Far:
    """One job whose cache has `pages` pages, of which the last ones are a small job's, and whose rows are the last of M."""

    def __init__(self, job, pages, M, row_names):
        persist, lane, sizes = job
        self.small, self.rows, self.names = job, sizes["M"], row_names
        self.page_bytes = 2 * sizes["Hkv"] * sizes["page"] * sizes["D"]
        self.first_page, self.M = pages - sizes["n_pages"], M
        lane = dict(lane, starts=(lane["starts"] + (M - self.rows)).astype(np.int32),
                    table=np.where(lane["table"] < sizes["n_pages"], lane["table"] + self.first_page, lane["table"]).astype(np.int32))
        self.sizes = dict(sizes, M=M, n_pages=pages)
        self.at, offs, total = {}, {}, 256
        for side, arrays in (("p", persist), ("l", lane)):
            at = 256
            for name, a in arrays.items():
                offs[name], size = at, a.nbytes
                if name in "kv":
                    size = pages * self.page_bytes
                elif name in row_names:
                    size = M * (a.nbytes // self.rows)
                at += up(size)
            offs[side] = at
            total += up(at)
        self.dp = DevicePool(total, policy=salus.POLICY_PACK)
        status, self.id = self.dp.pool.lane_alloc(offs.pop("p"), offs.pop("l"), 0, 0)
        assert status == salus.OK
        q = self.dp.pool.job_query(self.id)
        for name, a in list(persist.items()) + list(lane.items()):
            at = (q.persist_off if name in persist else q.lane_off) + offs[name]
            if name in "kv":
                at += self.first_page * self.page_bytes
            elif name in row_names:
                at += (M - self.rows) * (a.nbytes // self.rows)
            self.at[name] = at
            self.dp.write(at, a)
        self.off = {name + "_off": at for name, at in offs.items()}

    def read(self, _, name):
        a = {**self.small[0], **self.small[1]}[name]
        return self.dp.read(self.at[name], a.nbytes, a.dtype).reshape(a.shape).copy()


@pytest.mark.parametrize("seqs", [[(1, 300), (2, 70)], [(70, 200)]])
def test_attention_and_appends_behind_4_gib_of_cache(seqs):
    rng = np.random.default_rng(6)
    pages = (5 << 30) // (2 * 8 * 1024 * 256)
    far = Far(attention_job(rng, seqs, 8, 8, 256, 1024), pages, seqs[0][0] + sum(n for n, _ in seqs[1:]), ())
    descs, keep = salus.Pool.make_attention_descs([dict(far.sizes, job=far.id, **far.off)])
    assert far.dp.pool.grouped_attention(descs, stream=far.dp.stream) == salus.OK, far.dp.pool.last_error()
    far.dp.sync()
    check_attention(far, [far.small])
    far.dp.close()
    far = Far(append_job(rng, seqs, 8, 8, 256, 1024, 256, HALF), pages, sum(n for n, _ in seqs), ())
    descs, keep = salus.Pool.make_append_descs([dict(far.sizes, job=far.id, **far.off)])
    assert far.dp.pool.grouped_append(descs, stream=far.dp.stream) == salus.OK, far.dp.pool.last_error()
    far.dp.sync()
    check_append(far, [far.small])
    far.dp.close()


def test_rows_behind_4_gib():
    rng, M = np.random.default_rng(7), 1_100_000
    far = Far(attention_job(rng, [(3, 90), (1, 40)], 8, 1, 256, 32), 20, M, ("q", "y"))
    descs, keep = salus.Pool.make_attention_descs([dict(far.sizes, job=far.id, **far.off)])
    assert far.dp.pool.grouped_attention(descs, stream=far.dp.stream) == salus.OK, far.dp.pool.last_error()
    far.dp.sync()
    check_attention(far, [far.small])
    far.dp.close()
    far = Far(append_job(rng, [(11, 90), (1, 40)], 8, 1, 256, 32, 256, HALF), 20, M, ("x", "q"))
    descs, keep = salus.Pool.make_append_descs([dict(far.sizes, job=far.id, **far.off)])
    assert far.dp.pool.grouped_append(descs, stream=far.dp.stream) == salus.OK, far.dp.pool.last_error()
    far.dp.sync()
    check_append(far, [far.small])
    far.dp.close()


def test_logits_behind_4_gib():
    M, V = 48000, 50000
    rng = np.random.default_rng(8)
    params = [(1.0, 40, 0.9, 0.0), (0.9, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.02)]
    x = answer.bf16_values(bf16_bits(rng.standard_normal((4, V)) * 3)).astype(np.float32)
    _, lane, sizes = job = sample_job(x, params, rng.random(4), True)
    at, off = 256, {}
    for name, size in (("logits", M * V * 2), ("params", 16 * M), ("u", 4 * M), ("tokens", 4 * M), ("work", salus.sample_work_bytes(M, V))):
        off[name] = at
        at += up(size)
    dp = DevicePool(at + 4096, policy=salus.POLICY_PACK)
    status, id = dp.pool.lane_alloc(256, at, 0, 0)
    assert status == salus.OK
    base = dp.pool.job_query(id).lane_off
    dp.buf.zero_()                          # a temperature of zero: the first of equal logits
    dp.buf[base + off["tokens"]:base + off["tokens"] + 4 * M] = 0xff
    for name, a in lane.items():
        if name != "work":
            dp.write(base + off[name] + (M - 4) * (a.nbytes // 4), a)
    descs, keep = salus.Pool.make_sample_descs([dict(sizes, M=M, job=id, **{n + "_off": v for n, v in off.items()})])
    assert dp.pool.grouped_sample(descs, stream=dp.stream) == salus.OK, dp.pool.last_error()
    dp.sync()
    tokens = dp.read(base + off["tokens"], 4 * M, np.int32)

    class Last:
        def read(self, j, name):
            return tokens[-4:]
    check_sample(Last(), [job])
    assert (tokens[:-4] == 0).all()
    dp.close()
