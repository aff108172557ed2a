// Attention of new rows over the paged caches of a round's jobs: single tokens, or a few, of sequences of any length.
//
//   y = sum_t w_t v_t / sum_t w_t,  w_t = 2^(scale log2(e) q . k_t - m),  m the largest so far, sums scaled when it grows
//
// Bound by reading the cache once.  A workgroup takes sixteen columns, a key head and a part of the keys, its four wavefronts tiles of 32 keys by turns
// (v_mfma_f32_16x16x32_bf16); the parts of a long sequence are joined by a second kernel.
#include <algorithm>
#include <vector>

#include "attention_tile.hpp"

namespace salus {

constexpr uint32_t kAttentionThreads = 256, kFewColumns = 16;
constexpr int32_t kStride = 4 * (int32_t)kKeys;      // keys between two tiles of a wavefront

AttentionParts attention_parts(uint32_t M, uint32_t n_seqs, uint32_t Hq, uint32_t Hkv, uint32_t D, uint32_t max_len)
{
    const uint64_t tiles = (uint64_t)ColumnBase<kFewColumns>{Hq / Hkv}(M, n_seqs) * Hkv, target = 1024;
    const uint64_t part = std::max<uint64_t>(256, ((uint64_t)max_len * std::min(tiles, target) / target + 127) / 128 * 128);
    return {(uint32_t)part, (uint32_t)((max_len + part - 1) / part)};
}

// of the parts of a row: D sums, the largest score and the sum of the weights
uint64_t attention_work_floats(uint32_t M, uint32_t Hq, uint32_t D, const AttentionParts &parts)
{
    return parts.parts == 1 ? 0 : (uint64_t)M * Hq * parts.parts * (D + 2);
}

// A tile of 32 keys, D = 32 N elements a head.  Lane 16 g + c: of row c of K's fragment t, k-step i, elements 32 i + 8 g .. + 8 of key 8 (c / 4) + 4 t + c % 4;
// of V's fragment i element 16 i + c of tokens 8 g .. + 8.
template <int N>
struct FewTile {
    u32x4 k[N][2], v[2 * N];
    int32_t key;             // its first key
    bool seen;               // false: it lies in no page
};

template <int N>
struct FewLoads {
    static constexpr uint32_t D = 32 * N;
    const AttentionProblem &p;
    const Global<int32_t> *table;
    uint32_t head, k_at, v_at;
    int32_t first, end;          // this wavefront's first key, the part's end
    int32_t pages, pages_from;   // lane l: page of the tile that begins at pages_from + l kStride

    __device__ void load(int32_t key, FewTile<N> &t)
    {
        const uint32_t lane = threadIdx.x & 63;
        if (key >= pages_from + 64 * kStride) {
            pages_from = key;
            const uint32_t of = (uint32_t)(key + (int32_t)lane * kStride) >> p.seq.page_bits;
            pages = of < p.seq.max_pages ? table[of] : -1;
        }
        int32_t page = __builtin_amdgcn_readlane(pages, (uint32_t)(key - pages_from) / kStride);
        t.key = key;
        t.seen = page >= 0 && (uint32_t)page < p.seq.n_pages;
        if (!t.seen) page = 0;       // something to load
        const uint64_t from = (((uint64_t)page * p.seq.Hkv + head) << p.seq.page_bits) * (2 * D) + ((uint32_t)key & ((1u << p.seq.page_bits) - 1)) / 32 * (64 * D);
        const Global<char> *k = (const Global<char> *)p.k + from, *v = (const Global<char> *)p.v + from;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) t.k[i][u] = *(const Global<u32x4> *)(k + k_at + i * 2048 + u * 64);
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) t.v[i] = *(const Global<u32x4> *)(v + v_at + i * 256);
    }
};

// Running sums of sixteen columns: lane 16 g + c has elements 16 i + 4 g + e of column c in o[i][e], its share of l, and m.
template <int N>
struct FewSums {
    f32x4 o[2 * N];
    float m = -INFINITY, l = 0.0f;

    __device__ void scale_by(float f)
    {
        l *= f;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] *= f;
    }

    // all: every column sees every key of the tile.  end: the first key that none sees.
    __device__ void add(FewTile<N> &t, const u32x4 (&q)[N], float scale, Sight sight, bool all, int32_t end, const AttentionProblem &p, const FewLoads<N> &loads)
    {
        const uint32_t lane = threadIdx.x & 63, g = lane >> 4;
        f32x4 x[2] = {};
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) x[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_fragment(t.k[i][u]), as_fragment(q[i]), x[u], 0, 0, 0);
        const int32_t key = t.key + 8 * (int32_t)g;
        all = all && t.seen;
        if (!all) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!t.seen || !sight.sees(key + e)) x[e / 4][e % 4] = -INFINITY;
        }
        float top = x[0][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e / 4][e % 4]);
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float now = fmaxf(m, top * scale), base = now == -INFINITY ? 0.0f : now;
        if (__any(now != m)) scale_by(__builtin_amdgcn_exp2f(m - base));
        m = now;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float w = __builtin_amdgcn_exp2f(fmaf(x[e / 4][e % 4], scale, -base));
            x[e / 4][e % 4] = w;
            l += w;
        }
        if (!all) {
            // behind the last key the cache holds anything; among the keys, zero times a value that is no number would be none
            const int32_t left = t.seen ? end - key : 0;
            bool special = false;
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) {
                t.v[i] = first_tokens(t.v[i], left);
                special |= any_special(t.v[i]);
            }
            if (__any(special)) {
                add_seen(t, x, sight, p, loads);
                return;
            }
        }
        const u32x4 w = {bf16_pack(x[0][0], x[0][1]), bf16_pack(x[0][2], x[0][3]), bf16_pack(x[1][0], x[1][1]), bf16_pack(x[1][2], x[1][3])};
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_fragment(t.v[i]), as_fragment(w), o[i], 0, 0, 0);
    }

    // O^T += V^T P^T key by key, leaving out what a column does not see.  The values come from the lanes that hold them: element 16 i + 4 g + e of a key in
    // tokens 8 k .. + 8 is with lane 16 k + 4 g + e.
    __device__ void add_seen(const FewTile<N> &t, const f32x4 (&x)[2], Sight sight, const AttentionProblem &, const FewLoads<N> &)
    {
        const uint32_t lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
#pragma unroll 1
        for (uint32_t key = 0; key < kKeys; ++key) {
            const uint32_t owner = key / 8 * 16, part = key % 8;
            float w = x[0][0];
#pragma unroll
            for (uint32_t e = 1; e < 8; ++e) w = part == e ? x[e / 4][e % 4] : w;
            w = __shfl(w, owner + c, 64);
            const bool seen = t.seen && sight.sees(t.key + (int32_t)key);
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) {
                uint32_t pair = t.v[i][0];
#pragma unroll
                for (uint32_t e = 1; e < 4; ++e) pair = part / 2 == e ? t.v[i][e] : pair;
                const float mine = part % 2 ? bf16_high(pair) : bf16_low(pair);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = __shfl(mine, owner + 4 * g + e, 64);
                    if (seen) o[i][e] = fmaf(w, v, o[i][e]);
                }
            }
        }
    }
};

// N: D / 32.  TWO: a tile is asked for while the one before it is worked on.
template <int N, typename Args>
__global__ __launch_bounds__(kAttentionThreads, N <= 4 ? 2 : 1) void attend_few(Args a)
{
    constexpr uint32_t D = 32 * N;
    constexpr bool TWO = N <= 4;
    __shared__ float sums[2][kFewColumns][D];
    __shared__ float tops[2][kFewColumns], weights[2][kFewColumns];
    AttentionProblem p;
    const uint32_t t = find_owner(a.first, a.p, a.base + blockIdx.x, p);
    ColumnTile tile;
    if (!find_columns<kFewColumns>(p, t / p.parts, t % p.parts, tile) || tile.part >= max(tile.parts, 1u)) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
    const uint32_t G = p.seq.Hq / p.seq.Hkv, column = min(tile.first + c, tile.end - 1), i = column / G;
    const bool valid = tile.first + c < tile.end;
    const uint64_t row = (uint64_t)(tile.row + i) * p.seq.Hq + tile.head * G + column % G;
    u32x4 q[N];
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = *(const Global<u32x4> *)((const Global<char> *)p.q + row * (D * 2) + 64 * k + 16 * g);
    const Sight sight = sight_of(p, tile.position + (int32_t)i);
    // what all columns see
    const Sight every = {sight_of(p, tile.position + (int32_t)((tile.end - 1) / G)).low, tile.position + (int32_t)(tile.first / G)};

    FewSums<N> s;
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) s.o[k] = f32x4{};
    const int32_t from = tile.key + (int32_t)(tile.part * p.part), end = min(tile.key_end, from + (int32_t)p.part);
    FewLoads<N> loads{p, (const Global<int32_t> *)p.seq.table + (uint64_t)tile.s * p.seq.max_pages, tile.head,
                      (g * 32 + (c / 4) * 8 + c % 4) * 16, (g * D + c) * 16, from + (int32_t)(kKeys * wave), end, 0, INT32_MIN};
    const auto add = [&](FewTile<N> &tile_of) {
        const bool all = tile_of.key > every.low && tile_of.key + 31 <= every.high;
        s.add(tile_of, q, p.scale, sight, all, tile.key_end, p, loads);
    };
    if constexpr (TWO) {
        FewTile<N> one, two;
        int32_t key = loads.first;
        if (key < end) loads.load(key, one);
        while (key < end) {
            key += kStride;
            if (key < end) loads.load(key, two);
            add(one);
            if (key >= end) break;
            key += kStride;
            if (key < end) loads.load(key, one);
            add(two);
        }
    } else {
        FewTile<N> one;
        for (int32_t key = loads.first; key < end; key += kStride) {
            loads.load(key, one);
            add(one);
        }
    }
    s.l += __shfl_xor(s.l, 16, 64);
    s.l += __shfl_xor(s.l, 32, 64);

    // the four wavefronts' sums become one, in two steps
#pragma unroll
    for (uint32_t step = 2; step >= 1; step /= 2) {
        if (wave >= step && wave < 2 * step) {
            const uint32_t to = wave - step;
            if (g == 0) {
                tops[to][c] = s.m;
                weights[to][c] = s.l;
            }
#pragma unroll
            for (int k = 0; k < 2 * N; ++k) *(f32x4 *)&sums[to][c][16 * k + 4 * g] = s.o[k];
        }
        __syncthreads();
        if (wave < step) {
            const float other = tops[wave][c], m = fmaxf(s.m, other), f = rescale(other, m);
            s.scale_by(rescale(s.m, m));
            s.m = m;
            s.l = fmaf(weights[wave][c], f, s.l);
#pragma unroll
            for (int k = 0; k < 2 * N; ++k) {
                const f32x4 o = *(f32x4 *)&sums[wave][c][16 * k + 4 * g];
#pragma unroll
                for (int e = 0; e < 4; ++e) s.o[k][e] = fmaf(o[e], f, s.o[k][e]);
            }
        }
        __syncthreads();
    }
    if (wave != 0 || !valid) return;
    if (tile.parts > 1) {
        Global<float> *to = (Global<float> *)p.work + (row * p.parts + tile.part) * (D + 2);
        if (g == 0) {
            to[D] = s.m;
            to[D + 1] = s.l;
        }
#pragma unroll
        for (int k = 0; k < 2 * N; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) to[16 * k + 4 * g + e] = s.o[k][e];
        return;
    }
    const float f = s.l == 0.0f ? 0.0f : 1.0f / s.l;
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) {
        const u32x2 w = {bf16_pack(s.o[k][0] * f, s.o[k][1] * f), bf16_pack(s.o[k][2] * f, s.o[k][3] * f)};
        *(Global<u32x2> *)((Global<char> *)p.y + row * (D * 2) + (16 * k + 4 * g) * 2) = w;
    }
}

// The parts of every row that has several become one: a workgroup takes a tile of columns.
template <typename Args>
__global__ __launch_bounds__(kAttentionThreads) void join_parts(Args a)
{
    AttentionProblem p;
    const uint32_t t = find_owner(a.first, a.p, a.base + blockIdx.x, p);
    ColumnTile tile;
    if (!find_columns<kFewColumns>(p, t, 0, tile) || tile.parts < 2) return;
    const uint32_t D = p.seq.D, units = D / 2, G = p.seq.Hq / p.seq.Hkv;
    for (uint32_t at = threadIdx.x; at < (tile.end - tile.first) * units; at += kAttentionThreads) {
        const uint32_t column = tile.first + at / units, d = at % units * 2;
        const uint64_t row = (uint64_t)(tile.row + column / G) * p.seq.Hq + tile.head * G + column % G;
        const Global<float> *from = (const Global<float> *)p.work + row * p.parts * (D + 2);
        float m = -INFINITY, l = 0.0f, low = 0.0f, high = 0.0f;
        for (uint32_t i = 0; i < tile.parts; ++i) m = fmaxf(m, from[i * (D + 2) + D]);
        for (uint32_t i = 0; i < tile.parts; ++i) {
            const float f = rescale(from[i * (D + 2) + D], m);
            l = fmaf(from[i * (D + 2) + D + 1], f, l);
            low = fmaf(from[i * (D + 2) + d], f, low);
            high = fmaf(from[i * (D + 2) + d + 1], f, high);
        }
        const float f = l == 0.0f ? 0.0f : 1.0f / l;
        *(Global<uint32_t> *)((Global<char> *)p.y + row * (D * 2) + d * 2) = bf16_pack(low * f, high * f);
    }
}

namespace {

template <int N, uint32_t NP>
hipError_t launch_few(const AttentionProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    return launch_answer_of<AttentionProblem, NP>(attend_few<N>, kAttentionThreads, p, n, stream, launches,
                                                  [](const AttentionProblem &q) { return column_tiles<kFewColumns>(q) * q.parts; });
}

template <uint32_t NP>
hipError_t launch_all(const std::vector<AttentionProblem> *by_width, hipStream_t stream, uint64_t *launches)
{
    hipError_t e = hipSuccess;
    const auto run = [&](int width, hipError_t (*launch)(const AttentionProblem *, uint32_t, hipStream_t, uint64_t *)) {
        if (e == hipSuccess && !by_width[width].empty()) e = launch(by_width[width].data(), (uint32_t)by_width[width].size(), stream, launches);
    };
    run(1, launch_few<1, NP>);
    run(2, launch_few<2, NP>);
    run(3, launch_few<3, NP>);
    run(4, launch_few<4, NP>);
    run(6, launch_few<6, NP>);
    run(8, launch_few<8, NP>);
    return e;
}

}  // namespace

hipError_t launch_attention(const AttentionProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    std::vector<AttentionProblem> by_width[9], parted;
    for (uint32_t i = 0; i < n; ++i) {
        by_width[p[i].seq.D / 32].push_back(p[i]);
        if (p[i].parts > 1) parted.push_back(p[i]);
    }
    const hipError_t e = n <= kAnswerFew ? launch_all<kAnswerFew>(by_width, stream, launches) : launch_all<kAnswerProblems>(by_width, stream, launches);
    if (e != hipSuccess || parted.empty()) return e;
    const uint32_t count = (uint32_t)parted.size();
    if (count <= kAnswerFew)
        return launch_answer_of<AttentionProblem, kAnswerFew>(join_parts, kAttentionThreads, parted.data(), count, stream, launches, column_tiles<kFewColumns>);
    return launch_answer_of<AttentionProblem, kAnswerProblems>(join_parts, kAttentionThreads, parted.data(), count, stream, launches, column_tiles<kFewColumns>);
}

}  // namespace salus
