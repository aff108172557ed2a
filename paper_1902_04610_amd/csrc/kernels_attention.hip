// Attention of new rows over the paged caches of a round's jobs: single tokens, or a few, of sequences of any length.
//
//   y = sum_t w_t v_t / sum_t w_t,  w_t = 2^(scale log2(e) q . k_t - m),  m the largest so far, sums scaled when it grows
//
// Few rows: bound by reading the cache once (1.9 GB of two jobs' four sequences of 115000 keys 300 us, 6.3 TB/s; 285 MB of 90 sequences of 1 .. 6000 keys 75 us).  A workgroup takes sixteen columns, a key head and a part of the keys, its four wavefronts tiles of 32 keys by turns
// (v_mfma_f32_16x16x32_bf16); the parts of a long sequence are joined by a second kernel.
#include <algorithm>
#include <vector>

#include "attention_tile.hpp"

namespace salus {

constexpr uint32_t kAttentionThreads = 256, kFewColumns = 16;
// Columns of a sequence, on average, from which on tiles are large.  us of few / many with 16 32 64 128 256 512 columns: 16 sequences of 3000 keys, 8 key heads of 128,
// 40/52 55/57 72/62 109/56 194/120 342/182; with 4 8 16 32 64 128: 4 of 8000, 16 heads of 64, 28/43 27/35 29/44 34/36 67/48 111/69; 4 of 1000, 8 heads of 128,
// 14/23 14/24 15/24 16/19 17/22 26/24.
constexpr uint32_t kManyFrom = 64;
constexpr uint32_t many_waves(uint32_t D) { return D <= 128 ? 8 : 4; }
constexpr uint32_t many_columns(uint32_t D) { return 32 * many_waves(D); }
constexpr int32_t kStride = 4 * (int32_t)kKeys;      // keys between two tiles of a wavefront

// Few rows, one sequence of 8 key heads of 128, us for 500 / 1000 / 4000 / 16000 keys: parts of 256 10.6 11.1 11.4 19.9, of 512 8.4 12.3 12.6 18.9, of 1024 8.4
// 10.8 16.5 19.5: up to kWhole keys a second launch costs more than it saves.  16 such sequences, 1000 / 2000 keys: 18.5 28.9, 20.7 28.5, 16.2 32.6; 16 jobs,
// 90 sequences of 1 .. 6000 keys: 80, 67, 63.  The rule knows the job alone, not the call's others: what a job is answered does not depend on its neighbours.
// Prompts and chunks: a workgroup fills a compute unit, and what the rule cannot know (rows are a bound, jobs are several) makes more than one round of them likely.
// us with 512 / 256 / 192 workgroups wanted: chunks of 512 behind 8000 .. 20000 keys, a window of 4096, 102 96 78; of 512 behind 8000 120 96 107; a prompt of 2048 92 64
// 63; 256 behind 16000 58 75 81; 11 such shapes 0.91 and 0.88 of the time of 512.
// (Parts are asked for with kLeastPart keys at least; that many are then evened out and rounded up to 128: 1025 keys are three of 384.)
constexpr uint32_t kWhole = 1024, kLeastPart = 512, kFewTarget = 512, kManyTarget = 192;

AttentionParts attention_parts(uint32_t M, uint32_t n_seqs, uint32_t Hq, uint32_t Hkv, uint32_t D, uint32_t max_len, uint32_t window)
{
    const uint32_t G = Hq / Hkv;
    const bool many = (uint64_t)M * G >= (uint64_t)kManyFrom * n_seqs;
    const uint32_t columns = many ? many_columns(D) : kFewColumns;
    const uint64_t tiles = (uint64_t)ColumnBase{G, columns}(M, n_seqs) * Hkv;
    const auto part = [&](uint64_t keys) {
        if (keys <= kWhole) return (uint64_t)kWhole;
        const uint64_t target = many ? kManyTarget : kFewTarget, about = std::max<uint64_t>(kLeastPart, keys * std::min(tiles, target) / target), n = (keys + about - 1) / about;
        return ((keys + n - 1) / n + 127) / 128 * 128;
    };
    const auto parts = [](uint64_t keys, uint64_t of) { return (keys + of - 1) / of; };
    const uint64_t most = parts(max_len, part(max_len));      // what there is room for
    // with a window a tile's keys are no more than this
    const uint64_t keys = window ? std::min<uint64_t>(max_len, (uint64_t)window + columns / G + 32) : max_len;
    uint64_t of = part(keys);
    while (parts(keys, of) > most) of += 128;
    return {columns, (uint32_t)of, (uint32_t)parts(keys, of)};
}

// of the parts of a row: D sums, the largest score and the sum of the weights
uint64_t attention_work_floats(uint32_t M, uint32_t Hq, uint32_t D, const AttentionParts &parts)
{
    return parts.parts == 1 ? 0 : (uint64_t)M * Hq * parts.parts * (D + 2);
}

// What a call uses goes up and down with its rows, sequences and tokens: 64 rows of 32 heads of 128 behind 130000 tokens 14 MB, 63 of them 26, 4096 none.  A job's lane is
// laid out once, so its room is a bound that never falls.  With t tiles of c columns, T wanted: there are several parts only for t < T, no more than max_len / 512 rounded up and
// no more than (T / t) (513 / 512) + 1 (a part's keys are max_len t / T, rounded down where that is 512 or more); columns of all heads are fewer than c t.  So columns times
// parts are fewer than c T (513 / 512) + c t, and t is below T.
uint64_t attention_room_floats(uint32_t M, uint32_t Hq, uint32_t Hkv, uint32_t D, uint32_t max_len)
{
    if (max_len <= kWhole) return 0;
    const auto most = [](uint64_t columns, uint64_t target) { return columns * target * 1025 / 512; };
    uint64_t sums = most(kFewColumns, kFewTarget);
    if ((uint64_t)M * (Hq / Hkv) >= kManyFrom) sums = std::max(sums, most(many_columns(D), kManyTarget));
    return std::min(sums, (uint64_t)M * Hq * (((uint64_t)max_len + kLeastPart - 1) / kLeastPart)) * (D + 2);
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
    int32_t first;               // this wavefront's first key
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
        // read once: past the caches (306 us against 337 for 1.9 GB); keys, whose lines two loads share, through them
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) t.v[i] = __builtin_nontemporal_load((const Global<u32x4> *)(v + v_at + i * 256));
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
    __device__ void add(FewTile<N> &t, const u32x4 (&q)[N], float scale, Sight sight, bool all, int32_t end)
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
                add_seen(t, x, sight);
                return;
            }
        }
        const u32x4 w = {bf16_pack(x[0][0], x[0][1]), bf16_pack(x[0][2], x[0][3]), bf16_pack(x[1][0], x[1][1]), bf16_pack(x[1][2], x[1][3])};
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_fragment(t.v[i]), as_fragment(w), o[i], 0, 0, 0);
    }

    // O^T += V^T P^T key by key, leaving out what a column does not see.  The values come from the lanes that hold them: element 16 i + 4 g + e of a key in
    // tokens 8 k .. + 8 is with lane 16 k + 4 g + e.
    __device__ void add_seen(const FewTile<N> &t, const f32x4 (&x)[2], Sight sight)
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
    if (!find_columns<false>(p, t / p.parts, t % p.parts, tile) || tile.part >= max(tile.parts, 1u)) return;
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
                      (g * 32 + (c / 4) * 8 + c % 4) * 16, (g * D + c) * 16, from + (int32_t)(kKeys * wave), 0, INT32_MIN};
    const auto add = [&](FewTile<N> &tile_of) {
        const bool all = tile_of.key > every.low && tile_of.key + 31 <= every.high;
        s.add(tile_of, q, p.scale, sight, all, tile.key_end);
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

// ---- many rows ----------------------------------------------------------------------------------------------------------------
// Prompts and chunks of them: bound by the matrix pipes and by what the exponentials leave of them.  A workgroup's wavefronts have 32 columns each and share the tiles of keys and values, which
// travel straight into LDS, as they lie in the cache, two stages ahead (v_mfma_f32_32x32x16_bf16; every read from LDS is 512 consecutive bytes for each half of
// the lanes).  One barrier a stage: what it says is that all of the stage has landed and that the stage before it has been read.
// The largest score is only followed when it grows by more than 2^8 (lazy rescaling, a published method for running softmax sums): sums stay far below the largest float, and are
// scaled hardly ever.  Up to D = 128 the next tile's scores are multiplied while the weights of this one are made; from 192 on the sums leave no registers for that, and the two follow each other
// (4 jobs of 3 prompts of 2000 rows, 16 heads: 271 us at 128, 995 at 256).
// 12 prompts of 1000 - 2700 rows, 32 heads of 128: 465 us, 0.86 PFLOP/s; a tile of a wavefront takes some 950 cycles, 512 of them multiplies.
constexpr float kGrowth = 8.0f;

// Sixteen bytes a lane from base + from + off to LDS at `to` + 16 lane.  The scalars may come from lane reads: five wait states stand in front of their use.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void dma16_page(uint32_t to, uint64_t base, uint32_t from, uint32_t off)
{
    const u32x4 buffer = {(uint32_t)base, (uint32_t)(base >> 32) & 0xffffu, kOutside, 0x00027000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(buffer), "s"(from) : "m0", "memory");
}
#pragma clang diagnostic pop

// Bits 2 and 3 exchanged: row m of a fragment is key (or element of a value) swap_rows(m) of its 32, so that a lane's eight sums in a row are of consecutive ones.
__device__ inline uint32_t swap_rows(uint32_t m) { return (m & ~12u) | (m & 4u) << 1 | (m & 8u) >> 1; }

__device__ inline float larger_half(float x)      // of lanes l and l + 32
{
    const uint32_t w = __builtin_bit_cast(uint32_t, x);
    const auto both = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return fmaxf(as_float(both[0]), as_float(both[1]));
}

// Lane 32 h + c has of column c elements 32 i + 16 u + 8 h + e in o[i][8 u + e], and of a tile's scores those of keys 16 u + 8 h + e in x[8 u + e].
template <int N>
struct ManySums {
    static constexpr uint32_t D = 32 * N;
    f32x16 o[N];
    float m = -INFINITY, l = 0.0f;

    __device__ void follow(float top)
    {
        const float f = rescale(m, top);
        m = top;
        l *= f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] *= f;
    }

    // A lane's place in the fragments of keys and values.
    __device__ static uint32_t key_at() { return (threadIdx.x & 32) * 16 + swap_rows(threadIdx.x & 31) * 16; }
    __device__ static uint32_t value_at() { return (threadIdx.x & 32) / 32 * (D * 16) + swap_rows(threadIdx.x & 31) * 16; }

    // The queries' fragments: what registers do not hold (rest) is kept in LDS, where each lane finds its own.
    static constexpr int kHeld = N > 6 ? 12 : 2 * N, kRest = 2 * N - kHeld;

    __device__ static f32x16 scores(const char *k, const u32x4 (&q)[kHeld], const char *rest)
    {
        f32x16 x = {};
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) {
            const u32x4 mine = i < kHeld ? q[i < kHeld ? i : 0] : *(const u32x4 *)(rest + (i - kHeld) * 1024);
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8 *)(k + i * 1024), as_fragment(mine), x, 0, 0, 0);
            if constexpr (N > 6)
                if (i % 4 == 3) asm volatile("" ::: "memory");      // not all of them at once: there are no registers for them
        }
        return x;
    }

    __device__ static void hide(f32x16 &x, Sight sight, int32_t key_0, bool there)
    {
        const int32_t key = key_0 + (int32_t)(threadIdx.x & 32) / 4;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (!there || !sight.sees(key + 16 * (r / 8) + r % 8)) x[r] = -INFINITY;
    }

    // The largest score so far, of the column.
    __device__ float top_of(const f32x16 &x, float scale) const
    {
        float top = x[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
        return fmaxf(m, larger_half(top) * scale);
    }

    __device__ void weigh(f32x16 &x, float scale)
    {
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], scale, -base));
            l += x[r];
        }
    }
    __device__ static u32x4 packed(const f32x16 &x, int u)
    {
        return {bf16_pack(x[8 * u], x[8 * u + 1]), bf16_pack(x[8 * u + 2], x[8 * u + 3]), bf16_pack(x[8 * u + 4], x[8 * u + 5]), bf16_pack(x[8 * u + 6], x[8 * u + 7])};
    }
    __device__ static u32x4 value(const char *v, int i, int u) { return *(const u32x4 *)(v + (2 * u * D + 32 * i) * 16); }

    // O^T += V^T P^T.
    __device__ void add_values(const f32x16 &x, const char *v)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const u32x4 w = packed(x, u);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_fragment(value(v, i, u)), as_fragment(w), o[i], 0, 0, 0);
                if constexpr (N > 6) asm volatile("" ::: "memory");
            }
        }
    }

    // The same for a tile of which not every column sees every key.  v: where the tile's values begin.  end: the first key that no column of the wavefront sees.
    __device__ void add_seen_values(const f32x16 &x, const char *v, Sight sight, int32_t key_0, int32_t end)
    {
        const char *mine = v + value_at();
        const int32_t left = end - key_0 - (int32_t)(threadIdx.x & 32) / 4;
        const u32x4 meant[2] = {first_tokens(u32x4{~0u, ~0u, ~0u, ~0u}, left), first_tokens(u32x4{~0u, ~0u, ~0u, ~0u}, left - 16)};
        uint32_t carried = 0;      // an exponent of ones carries into the bit above it
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll N > 6 ? 1 : N
            for (int i = 0; i < N; ++i) {
                const u32x4 w = value(mine, i, u);
#pragma unroll
                for (int e = 0; e < 4; ++e) carried |= (w[e] & meant[u][e] & 0x7f807f80u) + 0x00800080u;
            }
        if (__any(carried & 0x80008000u)) {
            add_one_by_one(x, v, sight, key_0);
            return;
        }
        asm volatile("" ::: "memory");      // read again: there are no registers to keep them
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const u32x4 w = packed(x, u);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                u32x4 vs = value(mine, i, u);
#pragma unroll
                for (int e = 0; e < 4; ++e) vs[e] &= meant[u][e];
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_fragment(vs), as_fragment(w), o[i], 0, 0, 0);
                if constexpr (N > 6) asm volatile("" ::: "memory");
            }
        }
    }

    // O^T += V^T P^T key by key, leaving out what a column does not see.
    __device__ void add_one_by_one(const f32x16 &x, const char *v, Sight sight, int32_t key_0)
    {
        const uint32_t lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll 1
        for (uint32_t key = 0; key < kKeys; ++key) {
            float w = x[0];
#pragma unroll
            for (uint32_t r = 1; r < 16; ++r) w = key / 16 * 8 + key % 8 == r ? x[r] : w;
            w = __shfl(w, (lane & 31) + key / 8 % 2 * 32, 64);
            const bool seen = sight.sees(key_0 + (int32_t)key);
            if (!__any(seen)) continue;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float value = bf16_low(*(const uint16_t *)(v + (((key / 8) * D + 32 * i + 16 * (r / 8) + 8 * h + r % 8) * 8 + key % 8) * 2));
                    if (seen) o[i][r] = fmaf(w, value, o[i][r]);
                    if (r % 2 == 1) asm volatile("" ::: "memory");      // a few loads at a time: registers for all would be taken from the loop that matters
                }
        }
    }
};

template <int N, typename Args>
__global__ __launch_bounds__(64 * many_waves(32 * N), N == 1 ? 4 : many_waves(32 * N) / 4) void attend_many(Args a)
{
    // Tiles of a stage, stages that are asked for ahead; a stage is entered while the values of the tile in front of it are still to be read.
    constexpr uint32_t D = 32 * N, WAVES = many_waves(D), TILES = N <= 4 ? 4 : N == 6 ? 2 : 1, AHEAD = N <= 6 ? 1 : 2, RING = TILES * (1 + AHEAD) + 1;
    constexpr uint32_t kTile = 64 * D, kAsks = TILES * 2 * kTile / 1024 / WAVES;      // bytes of a tile's keys, or values; a wavefront's requests of 1 KB a stage
    __shared__ __attribute__((aligned(1024))) char smem[RING * 2 * kTile + WAVES * ManySums<N>::kRest * 1024];
    AttentionProblem p;
    const uint32_t t = find_owner(a.first, a.p, a.base + blockIdx.x, p);
    ColumnTile tile;
    if (!find_columns<true>(p, t / p.parts, t % p.parts, tile) || tile.part >= max(tile.parts, 1u)) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, c = lane & 31;
    const uint32_t G = p.seq.Hq / p.seq.Hkv, first = tile.first + 32 * wave, column = min(first + c, tile.end - 1), i = column / G;
    const bool valid = first + c < tile.end;
    const uint64_t row = (uint64_t)(tile.row + i) * p.seq.Hq + tile.head * G + column % G;
    using Sums = ManySums<N>;
    u32x4 q[Sums::kHeld];
    char *rest = smem + RING * 2 * kTile + wave * Sums::kRest * 1024 + lane * 16;
#pragma unroll
    for (int k = 0; k < 2 * N; ++k) {
        const u32x4 w = *(const Global<u32x4> *)((const Global<char> *)p.q + row * (D * 2) + 32 * k + 16 * h);
        if (k < Sums::kHeld) q[k < Sums::kHeld ? k : 0] = w;
        else *(u32x4 *)(rest + (k - Sums::kHeld) * 1024) = w;
    }
    const Sight sight = sight_of(p, tile.position + (int32_t)i);
    // what all columns of the wavefront see, and the keys between which any sees one
    const uint32_t last_row = (min(first + 32, tile.end) - 1) / G;
    const Sight every = {sight_of(p, tile.position + (int32_t)last_row).low, tile.position + (int32_t)(min(first, tile.end - 1) / G)};
    const int32_t none = first < tile.end ? tile.position + (int32_t)last_row + 1 : 0, low = sight_of(p, every.high).low;

    ManySums<N> s;
#pragma unroll
    for (int k = 0; k < N; ++k) s.o[k] = f32x16{};
    const int32_t from = tile.key + (int32_t)(tile.part * p.part), end = min(tile.key_end, from + (int32_t)p.part);
    const uint32_t tiles = end > from ? (uint32_t)(end - from + 31) / 32 : 0, stages = (tiles + TILES - 1) / TILES;
    const Global<int32_t> *table = (const Global<int32_t> *)p.seq.table + (uint64_t)tile.s * p.seq.max_pages;
    const uint32_t lds = lds_address(smem);
    // a stage is 2 TILES halves (a tile's keys, its values), each a share of the wavefronts'
    constexpr uint32_t kSharers = WAVES / (2 * TILES);
    const uint32_t half = wave / kSharers, share = wave % kSharers * kAsks;
    const uint64_t k_cache = (uint64_t)(uintptr_t)p.k, v_cache = (uint64_t)(uintptr_t)p.v, cache = half & 1 ? v_cache : k_cache;
    // lane l: page of tile (known + l), the ones that are asked for and the ones that are worked on
    int32_t pages = 0, pages_before = 0;
    uint32_t known = ~0u;
    bool missing = false;        // a page that is not there has been met
    const auto page_of = [&](uint32_t number) __attribute__((always_inline)) {
        return number >= known ? __builtin_amdgcn_readlane(pages, (number - known) & 63) : __builtin_amdgcn_readlane(pages_before, (number + 64 - known) & 63);
    };
    const auto there = [&](int32_t page) { return page >= 0 && (uint32_t)page < p.seq.n_pages; };
    // A stage's requests are made a few at a time: all at once they would keep every wavefront waiting until the addresses of most have been worked through.
    uint64_t ask_base = 0;
    uint32_t ask_to = 0, asked = kAsks;
    const auto aim = [&](uint32_t stage) __attribute__((always_inline)) {
        if (stage * TILES % 64 == 0) {
            pages_before = pages;
            known = stage * TILES;
            const uint32_t of = (uint32_t)(from + 32 * (int32_t)min(known + lane, tiles - 1)) >> p.seq.page_bits;
            pages = of < p.seq.max_pages ? table[of] : -1;
            missing = missing || __any(!there(pages));
            asm volatile("" : "+v"(pages));      // waited for here, where it is asked for: else the compiler waits, for all requests there are, wherever a page is looked up
        }
        const uint32_t place = stage * TILES + half / 2, number = min(place, tiles - 1), key = (uint32_t)from + 32 * number;
        int32_t page = page_of(number);
        if (!there(page)) page = 0;      // something to load: nobody looks at it
        ask_base = uniform64(cache + (((uint64_t)(uint32_t)page * p.seq.Hkv + tile.head) << p.seq.page_bits) * (2 * D) +
                             (uint64_t)((key & ((1u << p.seq.page_bits) - 1)) / 32) * kTile);
        ask_to = __builtin_amdgcn_readfirstlane(lds + (place % RING * 2 + (half & 1)) * kTile);
        asked = 0;
    };
    const auto ask = [&](uint32_t up_to) __attribute__((always_inline)) {
#pragma unroll 1
        for (; asked < min(up_to, kAsks); ++asked) dma16_page(ask_to + (share + asked) * 1024, ask_base, (share + asked) * 1024, lane * 16);
    };
    // A stage is there, and all wavefronts are through with what the next one that is asked for takes the place of.
    const auto enter = [&](uint32_t stage) __attribute__((always_inline)) {
        stage = __builtin_amdgcn_readfirstlane(stage);
        ask(kAsks);
        if (AHEAD > 1 && stage + 1 < stages) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - 1) * kAsks) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (stage + AHEAD < stages) aim(stage + AHEAD);
    };
    for (uint32_t stage = 0; stage < min(AHEAD, stages); ++stage) {
        aim(stage);
        ask(kAsks);
    }
    // this wavefront's tiles
    const int32_t seen_end = min(end, none);
    uint32_t n = low + 1 > from ? (uint32_t)(low + 1 - from) / 32 : 0;
    const uint32_t n_end = seen_end > from ? (uint32_t)(seen_end - from + 31) / 32 : 0;
    uint32_t entered = 0;
    const auto keys = [&](uint32_t number) { return smem + number % RING * (2 * kTile); };
    const auto key_of = [&](uint32_t number) { return from + 32 * (int32_t)number; };
    // tiles in front of this one are seen whole by all columns as far as the window goes
    const uint32_t whole_end = every.high + 1 > from ? min((uint32_t)(every.high + 1 - from) / 32, n_end) : 0;
    const auto whole = [&](uint32_t number) { return key_of(number) > every.low && key_of(number) + 31 <= every.high && there(page_of(number)); };
    if (n < n_end) {
        const uint32_t key_at = s.key_at(), value_at = s.value_at();
        for (; entered <= n / TILES; ++entered) enter(entered);
        f32x16 x = s.scores(keys(n) + key_at, q, rest);
        bool all = whole(n);
        if (!all) s.hide(x, sight, key_of(n), there(page_of(n)));
        float top = s.top_of(x, p.scale);
        if (__any(top > s.m)) s.follow(top);
        for (;;) {
            // Tiles that all columns see whole: the next tile's scores are multiplied while this one's weights are made, whose reads from LDS are asked for in front of both.
            bool grown = false;
            if constexpr (N <= 4) {
#pragma unroll 1
                while (all && n + 1 < whole_end && !missing) {
                    if ((n + 1) % TILES == 0) enter(entered++);
                    const char *k = keys(n + 1) + key_at, *v = keys(n) + kTile + value_at;
                    u32x4 ks[2 * N], vs[2][N], w[2];
#pragma unroll
                    for (int j = 0; j < 2 * N; ++j) ks[j] = *(const u32x4 *)(k + j * 1024);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int j = 0; j < N; ++j) vs[u][j] = s.value(v, j, u);
                    ask(asked + (kAsks + 2) / 3);
                    __builtin_amdgcn_sched_barrier(0);
                    s.weigh(x, p.scale);
                    w[0] = s.packed(x, 0);
                    w[1] = s.packed(x, 1);
                    f32x16 y = {};
#pragma unroll
                    for (int j = 0; j < 2 * N; ++j) y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_fragment(ks[j]), as_fragment(q[j]), y, 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int j = 0; j < N; ++j) s.o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_fragment(vs[u][j]), as_fragment(w[u]), s.o[j], 0, 0, 0);
                    x = y;
                    ++n;
                    top = s.top_of(x, p.scale);
                    grown = __any(top > s.m + kGrowth);
                    if (grown) break;
                }
            }
            if (grown) {
                s.follow(top);
                continue;
            }
            // the others, and the last one
            const bool more = n + 1 < n_end;
            if (more && (n + 1) % TILES == 0) enter(entered++);
            s.weigh(x, p.scale);
            if (all) s.add_values(x, keys(n) + kTile + value_at);
            else s.add_seen_values(x, keys(n) + kTile, sight, key_of(n), there(page_of(n)) ? none : 0);
            if (!more) break;
            ++n;
            x = s.scores(keys(n) + key_at, q, rest);
            all = whole(n);
            if (!all) s.hide(x, sight, key_of(n), there(page_of(n)));
            top = s.top_of(x, p.scale);
            if (__any(top > s.m + kGrowth)) s.follow(top);
        }
    }
    for (; entered < stages; ++entered) enter(entered);
    if (!valid) return;
    s.l += __shfl_xor(s.l, 32, 64);
    if (tile.parts > 1) {
        Global<float> *to = (Global<float> *)p.work + (row * p.parts + tile.part) * (D + 2);
        if (h == 0) {
            to[D] = s.m;
            to[D + 1] = s.l;
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) to[32 * k + 16 * (r / 8) + 8 * h + r % 8] = s.o[k][r];
        return;
    }
    const float f = s.l == 0.0f ? 0.0f : 1.0f / s.l;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = bf16_pack(s.o[k][8 * u + 2 * e] * f, s.o[k][8 * u + 2 * e + 1] * f);
            *(Global<u32x4> *)((Global<char> *)p.y + row * (D * 2) + (32 * k + 16 * u + 8 * h) * 2) = w;
        }
}

// The parts of every row that has several become one.  From 17 parts on a workgroup takes a column, its wavefronts a quarter of the parts each, its lanes the
// elements; below that it takes 16 columns, a thread four elements of one.
// 64 columns of 64 parts 6.6 us (16 with a wavefront to a column); 1088 columns of up to 12 parts 5.4 us; 32768 columns of 2 - 3 parts of 64 11.3 us.
constexpr uint32_t kFewParts = 16;
__host__ __device__ inline uint32_t join_columns(uint32_t parts) { return parts > kFewParts ? 1 : 16; }

__device__ inline void join_column(const AttentionProblem &p, uint64_t row, uint32_t parts, float (&sums)[4][256])
{
    constexpr uint32_t kAtOnce = 8;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = p.seq.D;
    const Global<float> *from = (const Global<float> *)p.work + row * p.parts * (D + 2);
    // each wavefront has the largest score of all parts, and the weights of its own: lane i of part begin + i
    float m = -INFINITY, l = 0.0f, sum[4] = {};
    for (uint32_t i = lane; i < parts; i += 64) m = fmaxf(m, from[(uint64_t)i * (D + 2) + D]);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    for (uint32_t i = lane; i < parts; i += 64) l = fmaf(from[(uint64_t)i * (D + 2) + D + 1], rescale(from[(uint64_t)i * (D + 2) + D], m), l);
    l = wave_total(l);
    const uint32_t begin = parts * wave / 4, end = parts * (wave + 1) / 4;
    for (uint32_t first = begin; first < end; first += 64) {
        const uint32_t n = min(end - first, 64u);
        const float top = from[(uint64_t)(first + min(lane, n - 1)) * (D + 2) + D], f = lane < n ? rescale(top, m) : 0.0f;
        for (uint32_t i = 0; i < n; i += kAtOnce) {
            float o[kAtOnce][4];
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j)
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) o[j][k] = i + j < n && lane + 64 * k < D ? from[(uint64_t)(first + i + j) * (D + 2) + lane + 64 * k] : 0.0f;
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j)
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) sum[k] = fmaf(o[j][k], i + j < n ? lane_value(f, (i + j) & 63) : 0.0f, sum[k]);
        }
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) sums[wave][lane + 64 * k] = sum[k];
    __syncthreads();
    const uint32_t e = threadIdx.x;
    if (e < D) {
        const float all = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
        ((Global<uint16_t> *)p.y)[row * D + e] = (uint16_t)bf16_bits(l == 0.0f ? 0.0f : all * (1.0f / l));
    }
}

template <typename Args>
__global__ __launch_bounds__(kAttentionThreads) void join_parts(Args a)
{
    __shared__ union {
        float share[16][kFewParts];             // of a part in its column
        float sums[4][256];
    } lds;
    AttentionProblem p;
    const uint32_t t = find_owner(a.first, a.p, a.base + blockIdx.x, p), each = join_columns(p.parts), pieces = p.columns / each;
    ColumnTile tile;
    if (!find_columns<false>(p, t / pieces, 0, tile) || tile.parts < 2) return;
    const uint32_t G = p.seq.Hq / p.seq.Hkv, D = p.seq.D, first = tile.first + t % pieces * each;
    if (first >= tile.end) return;
    const auto row_of = [&](uint32_t column) { return (uint64_t)(tile.row + column / G) * p.seq.Hq + tile.head * G + column % G; };
    if (each == 1) {
        join_column(p, row_of(first), tile.parts, lds.sums);
        return;
    }
    const uint32_t n = min(tile.end - first, 16u), stride = p.parts * (D + 2), i = threadIdx.x % 16;
    {
        const uint32_t c = threadIdx.x / 16;
        const Global<float> *of = (const Global<float> *)p.work + row_of(first + min(c, n - 1)) * stride + min(i, tile.parts - 1) * (D + 2) + D;
        const float top = of[0], weight = of[1];
        float m = top;
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
        const float f = i < tile.parts ? rescale(top, m) : 0.0f;
        float l = weight * f;
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) l += __shfl_xor(l, d, 64);
        lds.share[c][i] = l == 0.0f ? 0.0f : f / l;
    }
    __syncthreads();
    for (uint32_t at = threadIdx.x; at < n * (D / 4); at += kAttentionThreads) {
        const uint32_t c = at / (D / 4), e = at % (D / 4) * 4;
        const uint64_t row = row_of(first + c);
        const Global<float> *of = (const Global<float> *)p.work + row * stride + e;
        float sum[4] = {};
        for (uint32_t j = 0; j < tile.parts; j += 2) {
            const bool more = j + 1 < tile.parts;
            const Global<u32x2> *one = (const Global<u32x2> *)(of + j * (D + 2)), *two = (const Global<u32x2> *)(of + (j + more) * (D + 2));
            // zero times what is no number would be none
            const u32x2 none = {0u, 0u}, v[4] = {one[0], one[1], more ? two[0] : none, more ? two[1] : none};
            const float f = lds.share[c][j], h = more ? lds.share[c][j + 1] : 0.0f;
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) sum[k] = fmaf(as_float(v[2 + k / 2][k % 2]), h, fmaf(as_float(v[k / 2][k % 2]), f, sum[k]));
        }
        *(Global<u32x2> *)((Global<char> *)p.y + row * (D * 2) + e * 2) = u32x2{bf16_pack(sum[0], sum[1]), bf16_pack(sum[2], sum[3])};
    }
}

namespace {

template <int N, uint32_t NP>
hipError_t launch_width(const AttentionProblem *p, uint32_t n, bool many, hipStream_t stream, uint64_t *launches)
{
    const auto tiles = [](const AttentionProblem &q) { return column_tiles(q) * q.parts; };
    if (many) return launch_answer_of<AttentionProblem, NP>(attend_many<N>, 64 * many_waves(32 * N), p, n, stream, launches, tiles);
    return launch_answer_of<AttentionProblem, NP>(attend_few<N>, kAttentionThreads, p, n, stream, launches, tiles);
}

template <uint32_t NP>
hipError_t launch_parts(const AttentionProblem *p, uint32_t n, uint32_t width, bool many, hipStream_t stream, uint64_t *launches)
{
    switch (width) {
    case 32: return launch_width<1, NP>(p, n, many, stream, launches);
    case 64: return launch_width<2, NP>(p, n, many, stream, launches);
    case 96: return launch_width<3, NP>(p, n, many, stream, launches);
    case 128: return launch_width<4, NP>(p, n, many, stream, launches);
    case 192: return launch_width<6, NP>(p, n, many, stream, launches);
    default: return launch_width<8, NP>(p, n, many, stream, launches);
    }
}

}  // namespace

hipError_t launch_attention(const AttentionProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    // a launch for each width and kind that is there
    std::vector<AttentionProblem> group;
    group.reserve(n);
    for (uint32_t width = 32; width <= 256; width += 32)
        for (int many = 0; many < 2; ++many) {
            group.clear();
            for (uint32_t i = 0; i < n; ++i)
                if (p[i].seq.D == width && (p[i].columns != kFewColumns) == (many != 0)) group.push_back(p[i]);
            if (group.empty()) continue;
            const uint32_t count = (uint32_t)group.size();
            const hipError_t e = count <= kAnswerFew ? launch_parts<kAnswerFew>(group.data(), count, width, many, stream, launches)
                                                     : launch_parts<kAnswerProblems>(group.data(), count, width, many, stream, launches);
            if (e != hipSuccess) return e;
        }
    group.clear();
    for (uint32_t i = 0; i < n; ++i)
        if (p[i].parts > 1) group.push_back(p[i]);
    const uint32_t count = (uint32_t)group.size();
    if (count == 0) return hipSuccess;
    const auto pieces = [](const AttentionProblem &q) { return column_tiles(q) * (q.columns / join_columns(q.parts)); };
    if (count <= kAnswerFew) return launch_answer_of<AttentionProblem, kAnswerFew>(join_parts, kAttentionThreads, group.data(), count, stream, launches, pieces);
    return launch_answer_of<AttentionProblem, kAnswerProblems>(join_parts, kAttentionThreads, group.data(), count, stream, launches, pieces);
}

}  // namespace salus
