// Pieces of the transformer-block kernels (gated feed-forward blocks, dense layers with bias and residual, and their
// gradients): the by-value argument block, the activations with their slopes, and what becomes of a tile's sums on their way
// to memory.
#pragma once
#include "tile_mfma.hpp"

namespace salus {

// One job's product and its epilogue.
struct BlockProblem {
    const void *W;       // dense, gated: K x N (gated: K x 2 N, the gate's columns in front of the other half's); transposed: N x K
    const void *X;       // M x K bf16
    void *Y;             // M x N (gate gradient: M x 2 N)
    const void *R;       // dense: M x N bf16 added in front of the rounding, or null
    float *Z;            // dense, gated: M x N (M x 2 N) floats in front of the activation, written if not null; gate gradient: read
    const void *B;       // dense: N bf16 added in front of the activation, or null
    uint32_t M, K, N;
    uint32_t flags;      // bits 0-7 activation; kOutBf16, kReadAgain
};
constexpr uint32_t kReadAgain = 1u << 16;    // for the launcher: a backward pass will read W again
constexpr uint32_t kBlockProblems = 56;      // of a launch
struct BlockArgs {
    uint32_t n, tiles, base, pad;            // base: kernels of one tile per workgroup begin with this one
    uint32_t first[kBlockProblems];          // first tile of problem i; kNoTile from n on
    BlockProblem p[kBlockProblems];
};
static_assert(sizeof(BlockArgs) <= 4096, "kernel arguments are limited to 4 KB");
// The same for launches of few problems, whose time is the host's.
constexpr uint32_t kBlockFew = 4;
struct BlockFewArgs {
    uint32_t n, tiles, base, pad;
    uint32_t first[kBlockFew];
    BlockProblem p[kBlockFew];
};

// A grid has fewer than 2^32 threads: kernels of one tile per workgroup, of `threads` threads (a power of two), take more tiles in several launches (of a multiple of 8, for
// the XCDs).  launch(workgroups, first tile).
constexpr uint64_t kMostThreads = 1u << 31;
template <typename Launch>
inline hipError_t launch_tiles(uint64_t tiles, int threads, uint64_t *launches, Launch launch)
{
    const uint64_t most = kMostThreads / threads;
    for (uint64_t base = 0; base < tiles; base += most) {
        launch((uint32_t)(tiles - base < most ? tiles - base : most), (uint32_t)base);
        if (launches) *launches += 1;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// What a product's sums become: Y = act(X W + B) + R; Y = act(X Wg) * (X Wu); [dG dU] of dH = X W^T; X W^T itself.
enum class Epilogue { kDense, kGated, kGateGrad, kPlainT };

// ---- activations ------------------------------------------------------------------------------------------------------------
// NaNs pass through all of them and their slopes, as they do through the products: a gradient of what is no number is none.
// Upper tail of the normal distribution at c in [0, 9]: 2^p(c), p the polynomial of degree 8 that minimizes the largest c |2^p - Q| over [0, 6]
// (1e-8; fitted by linear programming), so Phi is off by 1.3e-7.  GELU(z) is z Q for negative z and z - z Q for others: max(z, 0) - |z| Q,
// which subtracts nothing from a negative z's small result.  (The library's erfc takes four times as long: 24 jobs x 1 - 128 rows,
// 1000 -> 3080, float results, 9 of 49 us.)  gelu_fast, two degrees less, suffices where a bf16 is next.
__device__ inline float tail_exponent(float c)
{
    float p = fmaf(-1.8847762248697109e-06f, c, 2.7810900064650923e-05f);
    p = fmaf(p, c, -0.00013004051288589835f);
    p = fmaf(p, c, -0.0002765035897027701f);
    p = fmaf(p, c, 0.007253301329910755f);
    p = fmaf(p, c, -0.0526358038187027f);
    p = fmaf(p, c, -0.4591573178768158f);
    p = fmaf(p, c, -1.15111243724823f);
    return fmaf(p, c, -0.9999998211860657f);
}
__device__ inline float normal_tail(float c) { return __builtin_amdgcn_exp2f(tail_exponent(c)); }
// The same at c in [0, 13] for results that stay floats: from 3.25 on, where an absolute error of Q is no small part of it any more, the polynomial
// of degree 7 that minimizes the largest |p - log2 Q| over [3.25, 13].  GELU of it is off by less than 1.2e-7 of |z|, and for negative z by less
// than 2.1e-5 of itself down to -12.9, where it is 3e-37 (in float arithmetic).  24 jobs x 1 - 128 rows as above, from the cache, 31.0 us with
// one polynomial, 32.0 with both.
__device__ inline float normal_tail_far(float c)
{
    float p = fmaf(-6.624220816320303e-08f, c, 4.464800895220833e-06f);
    p = fmaf(p, c, -0.00013070812565274537f);
    p = fmaf(p, c, 0.0021917573176324368f);
    p = fmaf(p, c, -0.02350013330578804f);
    p = fmaf(p, c, -0.5481355786323547f);
    p = fmaf(p, c, -1.0025348663330078f);
    p = fmaf(p, c, -1.106598138809204f);
    return __builtin_amdgcn_exp2f(c < 3.25f ? tail_exponent(c) : p);
}
// exp's argument is off by 2^-24 of itself, which the slope of the sigmoid takes back: 3e-8 of |z| at most in z sigmoid(z), beside the last bits of
// v_exp_f32 and v_rcp_f32.
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z)); }
__device__ inline float relu_nan(float z) { return z < 0.0f ? 0.0f : z; }

// `fine`: for results that stay floats.
template <int N>
__device__ inline void activate_all(float (&z)[N], uint32_t act, bool fine)
{
    if (act == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = relu_nan(z[i]);
    } else if (act == 2 && fine) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float c = fminf(fabsf(z[i]), 13.0f);      // beyond it, also at an infinity, nothing is left of a negative z
            z[i] = fmaf(-c, normal_tail_far(c), relu_nan(z[i]));
        }
    } else if (act == 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = gelu_fast(z[i]);
    } else if (act == 3) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] * sigmoid(z[i]);
    }
}

// a = act(z), d = act'(z): GELU'(z) = Phi(z) + z phi(z), SiLU'(z) = s (1 + z (1 - s)), s = sigmoid(z).
template <int N>
__device__ inline void activate_with_slope(const float (&z)[N], float (&a)[N], float (&d)[N], uint32_t act)
{
    if (act == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] = relu_nan(z[i]);
            d[i] = z[i] > 0.0f ? 1.0f : z[i] <= 0.0f ? 0.0f : z[i];
        }
    } else if (act == 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float c = fminf(fabsf(z[i]), 9.0f), q = normal_tail(c);
            const float phi = 0.39894228040143267794f * __builtin_amdgcn_exp2f(-0.72134752f * z[i] * z[i]);
            a[i] = fmaf(-c, q, relu_nan(z[i]));
            d[i] = fmaf(z[i], phi, z[i] < 0.0f ? q : 1.0f - q);
        }
    } else if (act == 3) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = sigmoid(z[i]);
            a[i] = z[i] * s;
            d[i] = s * fmaf(z[i], 1.0f - s, 1.0f);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] = z[i];
            d[i] = 1.0f;
        }
    }
}

// ---- sums on their way to memory ----------------------------------------------------------------------------------------------
__device__ inline float as_float(uint32_t w) { return __builtin_bit_cast(float, w); }      // (of a vector's element the builtin takes the first)
__device__ inline float bf16_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf16_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

// A 32 x 32 block in line order (to_lines_f32): of row 8 q + l % 8, lane l has the four columns line_column_f32(l) .. + 3.
typedef float Lines[4][4];      // [q][column]
__device__ inline void to_lines(const float (&v)[16], Lines &o)
{
    f32x4 lines[2][2];
    to_lines_f32(v, lines);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[q][e] = lines[q >> 1][q & 1][e];
}
// Two such blocks side by side as bf16, exchanged across the halves of the wavefront: a lane then has eight columns, pair_column(l) ..
// + 7, of the block l / 32, and eight lanes a whole line.
__device__ inline uint32_t pair_column(int lane) { return 32u * (lane >> 5) + 16u * ((lane >> 3) & 1u) + 8u * ((lane >> 4) & 1u); }
__device__ inline u32x4 pair_up(const float (&a)[4], const float (&b)[4])
{
    uint32_t a0 = bf16_pack(a[0], a[1]), a1 = bf16_pack(a[2], a[3]), b0 = bf16_pack(b[0], b[1]), b1 = bf16_pack(b[2], b[3]);
    swap_halves(a0, b0);
    swap_halves(a1, b1);
    return u32x4{a0, a1, b0, b1};
}

// Where a wavefront's part of a tile lies: its first row and column, and how many of each the matrix has from there on.
struct Part {
    uint32_t m, n, rows, cols;
    __device__ Part(const BlockProblem &p, uint32_t m_, uint32_t n_) : m(m_), n(n_), rows(m_ < p.M ? p.M - m_ : 0), cols(n_ < p.N ? p.N - n_ : 0) {}
};

__device__ inline void store4(float *at, const float (&v)[4]) { *(f32x4 *)at = f32x4{v[0], v[1], v[2], v[3]}; }

// J blocks of rows r0 .. + 31, columns c0 .. (of the part), row-major with `pitch` elements, rounded to bf16.
template <int J>
__device__ inline void store_bf16(uint16_t *Y, uint32_t pitch, const Part &at, uint32_t r0, uint32_t c0, const Lines (&o)[J], int lane)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t r = r0 + 8u * q + (lane & 7);
        if constexpr (J == 2) {
            const u32x4 w = pair_up(o[0][q], o[1][q]);
            const uint32_t c = c0 + pair_column(lane);
            if (r < at.rows && c < at.cols) *(u32x4 *)(Y + (size_t)r * pitch + c) = w;
        } else {
            const uint32_t c = c0 + line_column_f32(lane);
            if (r < at.rows && c < at.cols) *(u32x2 *)(Y + (size_t)r * pitch + c) = u32x2{bf16_pack(o[0][q][0], o[0][q][1]), bf16_pack(o[0][q][2], o[0][q][3])};
        }
    }
}

// act(sums + B) + R; the sums with B to Z.  N is a multiple of 8, so a vector of up to 8 columns lies wholly inside or outside.
// EARLY: R is asked for before the activations and used behind them, where there are registers for that.
template <int J, bool EARLY>
__device__ inline void finish_dense(const BlockProblem &p, const Part &at, uint32_t r0, uint32_t c0, const float (&v)[J][16], int lane)
{
    const uint32_t N = p.N, act = p.flags & 0xffu, column = line_column_f32(lane);
    const uint64_t corner = (uint64_t)at.m * N + at.n;
    const bool out_bf16 = (p.flags & kOutBf16) != 0;
    const uint16_t *R = (const uint16_t *)p.R + corner;
    uint32_t wide[4][4];
    u32x2 narrow[J][4];
    auto ask_residual = [&]() {
        if (!p.R) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t r = r0 + 8u * q + (lane & 7);
            if (J == 2 && out_bf16) {
                const uint32_t c = c0 + pair_column(lane);
                const u32x4 w = r < at.rows && c < at.cols ? *(const u32x4 *)(R + (size_t)r * N + c) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                for (int d = 0; d < 4; ++d) wide[q][d] = w[d];
            } else {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const uint32_t c = c0 + 32u * j + column;
                    narrow[j][q] = r < at.rows && c < at.cols ? *(const u32x2 *)(R + (size_t)r * N + c) : u32x2{0u, 0u};
                }
            }
        }
    };
    if (EARLY) ask_residual();
    Lines o[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        to_lines(v[j], o[j]);
        const uint32_t c = c0 + 32u * j + column;
        if (p.B) {
            const u32x2 b = c < at.cols ? *(const u32x2 *)((const uint16_t *)p.B + at.n + c) : u32x2{0u, 0u};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                o[j][q][0] += bf16_low(b[0]);
                o[j][q][1] += bf16_high(b[0]);
                o[j][q][2] += bf16_low(b[1]);
                o[j][q][3] += bf16_high(b[1]);
            }
        }
        if (p.Z) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t r = r0 + 8u * q + (lane & 7);
                if (r < at.rows && c < at.cols) store4(p.Z + corner + (size_t)r * N + c, o[j][q]);
            }
        }
        activate_all(*(float (*)[16])&o[j], act, !out_bf16);
    }
    if (!EARLY) ask_residual();
    if (p.R) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (J == 2 && out_bf16) {
                swap_halves(wide[q][0], wide[q][2]);      // back to four columns of each block
                swap_halves(wide[q][1], wide[q][3]);
                narrow[0][q] = u32x2{wide[q][0], wide[q][1]};
                narrow[J - 1][q] = u32x2{wide[q][2], wide[q][3]};
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                o[j][q][0] += bf16_low(narrow[j][q][0]);
                o[j][q][1] += bf16_high(narrow[j][q][0]);
                o[j][q][2] += bf16_low(narrow[j][q][1]);
                o[j][q][3] += bf16_high(narrow[j][q][1]);
            }
        }
    }
    if (out_bf16) {
        store_bf16<J>((uint16_t *)p.Y + corner, N, at, r0, c0, o, lane);
        return;
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t r = r0 + 8u * q + (lane & 7), c = c0 + 32u * j + column;
            if (r < at.rows && c < at.cols) store4((float *)p.Y + corner + (size_t)r * N + c, o[j][q]);
        }
}

// act(g) * u of J blocks of each; g and u to Z, beside each other as they lie in the weights.  The product is rounded to bf16 because it is a factor of
// the second product, which the matrix pipes take as bf16: up to half a step, 2^-8, of each hidden activation, 1.7e-3 of the
// results' size on average, as much as their own rounding.  g and u stay floats.
template <int J>
__device__ inline void finish_gated(const BlockProblem &p, const Part &at, uint32_t r0, uint32_t c0, const float (&g)[J][16],
                                    const float (&u)[J][16], int lane)
{
    const uint32_t N = p.N, column = line_column_f32(lane);
    Lines h[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        Lines up;
        to_lines(g[j], h[j]);
        to_lines(u[j], up);
        if (p.Z) {
            const uint32_t c = c0 + 32u * j + column;
            float *Z = p.Z + (uint64_t)at.m * (2 * N) + at.n + c;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t r = r0 + 8u * q + (lane & 7);
                if (!(r < at.rows && c < at.cols)) continue;
                store4(Z + (size_t)r * (2 * N), h[j][q]);
                store4(Z + (size_t)r * (2 * N) + N, up[q]);
            }
        }
        activate_all(*(float (*)[16])&h[j], p.flags & 0xffu, false);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) h[j][q][e] *= up[q][e];
    }
    store_bf16<J>((uint16_t *)p.Y + (uint64_t)at.m * N + at.n, N, at, r0, c0, h, lane);
}

// dG = dH * u * act'(g) and dU = dH * act(g), beside each other, of J blocks of dH; rounded to bf16 as factors of dX and dWin.  Eight rows at a time, the next eight asked for
// meanwhile: more of g and u does not fit beside the sums of a large tile.
template <int J>
__device__ inline void finish_gate_grad(const BlockProblem &p, const Part &at, uint32_t r0, uint32_t c0, const float (&v)[J][16], int lane)
{
    const uint32_t N = p.N, column = line_column_f32(lane);
    const float *Z = p.Z + (uint64_t)at.m * (2 * N) + at.n;
    uint16_t *Y = (uint16_t *)p.Y + (uint64_t)at.m * (2 * N) + at.n;
    f32x4 g[2][J], u[2][J];
    auto load = [&](int q) {
        const uint32_t r = r0 + 8u * q + (lane & 7);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const uint32_t c = c0 + 32u * j + column;
            const bool in = r < at.rows && c < at.cols;
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            g[q & 1][j] = in ? *(const f32x4 *)(Z + (size_t)r * (2 * N) + c) : zero;
            u[q & 1][j] = in ? *(const f32x4 *)(Z + (size_t)r * (2 * N) + N + c) : zero;
        }
    };
    load(0);
    Lines dh[J];
#pragma unroll
    for (int j = 0; j < J; ++j) to_lines(v[j], dh[j]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q < 3) load(q + 1);
        __builtin_amdgcn_sched_barrier(0);
        float z[4 * J], du[J][4], dg[J][4];
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * j + e] = g[q & 1][j][e];
        activate_with_slope(z, *(float (*)[4 * J])&du, *(float (*)[4 * J])&dg, p.flags & 0xffu);
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                du[j][e] *= dh[j][q][e];
                dg[j][e] *= dh[j][q][e] * u[q & 1][j][e];
            }
        const uint32_t r = r0 + 8u * q + (lane & 7), c = c0 + (J == 2 ? pair_column(lane) : column);
        const bool in = r < at.rows && c < at.cols;
        uint16_t *to = Y + (size_t)r * (2 * N) + c;
        if constexpr (J == 2) {
            const u32x4 wg = pair_up(dg[0], dg[1]), wu = pair_up(du[0], du[1]);
            if (in) {
                *(u32x4 *)to = wg;
                *(u32x4 *)(to + N) = wu;
            }
        } else if (in) {
            *(u32x2 *)to = u32x2{bf16_pack(dg[0][0], dg[0][1]), bf16_pack(dg[0][2], dg[0][3])};
            *(u32x2 *)(to + N) = u32x2{bf16_pack(du[0][0], du[0][1]), bf16_pack(du[0][2], du[0][3])};
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// ---- tile walks (tile_mfma.hpp) ---------------------------------------------------------------------------------------------------
// Gated: a tile of BN columns is BN / 2 of the gate's and the same BN / 2 of the other half's, sixteen and sixteen by turns
// (OperandStream's PAIRS), so that a lane has a gate's sum and its partner's in registers r and r + 8 of one block.
template <int BM, int BN, Epilogue E, typename Args = BlockArgs>
struct BlockWalk {
    static constexpr uint32_t kProblems = sizeof(Args::first) / 4;
    static constexpr uint32_t kCols = E == Epilogue::kGated ? BN / 2 : BN;      // of the output
    static constexpr bool kTransposed = E == Epilogue::kGateGrad || E == Epilogue::kPlainT;
    const Args &a;
    const uint32_t first;      // lane i: the first tile of problem i
    struct Place { int problem; uint32_t m0, n0, depth; };
    __device__ explicit BlockWalk(const Args &args) : a(args), first(args.first[min(threadIdx.x & 63, kProblems - 1)]) {}
    __device__ uint32_t tiles() const { return a.tiles; }
    // Tiles of one job in bands of 8 row tiles, column tiles inside a band: the tiles an XCD runs at a time then share 8
    // slabs of X and 4 - 8 slabs of W in its L2.
    __device__ Place place(uint32_t tile_id) const
    {
        const uint32_t id = xcd_remap(tile_id, a.tiles);
        const int g = __builtin_amdgcn_readfirstlane(wave_find_range(first, id, (threadIdx.x & 63) < kProblems));
        const BlockProblem &p = a.p[g];
        const uint32_t t = id - __builtin_amdgcn_readlane(first, g), rt = (p.M + BM - 1) / BM, ct = (p.N + kCols - 1) / kCols;
        const uint32_t band = t / (8u * ct), local = t - band * 8u * ct, rows = min(8u, rt - band * 8u);
        return {g, (band * 8u + local % rows) * BM, (local / rows) * kCols, p.K};
    }
    __device__ Operand m(const Place &at) const
    {
        const BlockProblem &p = a.p[at.problem];
        return {p.X, p.K, p.M, p.K * 2u, false};
    }
    __device__ Operand n(const Place &at) const
    {
        const BlockProblem &p = a.p[at.problem];
        if (kTransposed) return {p.W, p.K, p.N, p.K * 2u, false};
        if (E == Epilogue::kGated) return {p.W, p.K, p.N, p.N * 4u, false, p.N * 2u};
        return {p.W, p.K, p.N, p.N * 2u, false};
    }
    struct Held {};
    __device__ void begin(const Place &, Held &, uint32_t, uint32_t, int) const {}
    template <int FN, int FM, typename Landed>
    __device__ void finish(const Place &place, const f32x16 (&acc)[FN][FM], const Held &, uint32_t m, uint32_t n, int lane, Landed landed) const
    {
        const BlockProblem &p = a.p[place.problem];
        constexpr bool kGated = E == Epilogue::kGated;
        static_assert(!kGated || FN % 2 == 0, "two blocks of sums make one of results");
        constexpr int kBlocks = kGated ? FN / 2 : FN, J = kBlocks % 2 == 0 ? 2 : 1;
        const Part at(p, place.m0 + m, place.n0 + (kGated ? n / 2 : n));
        landed();
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < kBlocks; j += J) {
                __builtin_amdgcn_sched_barrier(0);       // one line at a time: the accumulators leave few registers
                if constexpr (kGated) {
                    float g[J][16], u[J][16];
#pragma unroll
                    for (int jj = 0; jj < J; ++jj)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const f32x16 &s = acc[2 * (j + jj) + (r >> 3)][i];
                            g[jj][r] = s[r & 7];
                            u[jj][r] = s[8 + (r & 7)];
                        }
                    finish_gated<J>(p, at, 32u * i, 32u * j, g, u, lane);
                } else {
                    float v[J][16];
#pragma unroll
                    for (int jj = 0; jj < J; ++jj)
#pragma unroll
                        for (int r = 0; r < 16; ++r) v[jj][r] = acc[j + jj][i][r];
                    if constexpr (E == Epilogue::kGateGrad) {
                        finish_gate_grad<J>(p, at, 32u * i, 32u * j, v, lane);
                    } else if constexpr (E == Epilogue::kPlainT) {
                        Lines o[J];
#pragma unroll
                        for (int jj = 0; jj < J; ++jj) to_lines(v[jj], o[jj]);
                        store_bf16<J>((uint16_t *)p.Y + (uint64_t)at.m * p.N + at.n, p.N, at, 32u * i, 32u * j, o, lane);
                    } else {
                        finish_dense<J, FM * FN <= 4>(p, at, 32u * i, 32u * j, v, lane);
                    }
                }
            }
    }
};

// ---- launchers ----------------------------------------------------------------------------------------------------------------
// All n problems, of any sizes.  cached: as for launch_grouped_bf16.
hipError_t launch_block_dense(const BlockProblem *p, uint32_t n, bool cached, hipStream_t stream, uint64_t *launches);
hipError_t launch_block_gated(const BlockProblem *p, uint32_t n, bool cached, hipStream_t stream, uint64_t *launches);
hipError_t launch_block_gate_grad(const BlockProblem *p, uint32_t n, bool cached, hipStream_t stream, uint64_t *launches);

// dZ = dY * act'(Z) of a dense layer, and the column sums of it: db itself for up to kSlopeRows rows, else those of blocks of as many.
struct SlopeProblem {
    const void *dY;      // M x N bf16
    const float *Z;      // M x N, or null (no activation)
    void *dZ;            // M x N bf16, or null (not wanted: dZ is dY)
    float *partial;      // column sums of blocks of kSlopeRows rows, ceil(M / kSlopeRows) x N; may be null if db is
    float *db;           // N floats, or null
    uint32_t M, N, act;
};
constexpr uint32_t kSlopeRows = 16;
hipError_t launch_block_slope(const SlopeProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches);

// dW = X^T . G.
struct WeightGradProblem {
    const void *X;       // M x K bf16
    const void *G;       // M x N bf16
    void *dW;            // K x N bf16
    uint32_t M, K, N;
};
// What a backward pass ends with, none of which waits for another: input gradients (BlockProblem as for a transposed product), weight gradients and the
// column sums that launch_block_slope left (db of jobs of more than kSlopeRows rows).  Any of the counts may be zero.
hipError_t launch_gradients(const BlockProblem *input, uint32_t n_input, const WeightGradProblem *weight, uint32_t n_weight, const SlopeProblem *sums, uint32_t n_sums,
                            bool cached, hipStream_t stream, uint64_t *launches);

// ---- gradient clipping ------------------------------------------------------------------------------------------------------------
struct ClipTensor {
    void *g;             // count elements of `dtype`
    float *wm;           // clip_sgd: float weights and their bf16 copy
    void *wb;
    uint64_t count;
    int32_t bf16;
};
struct ClipJob {
    const ClipTensor *tensors;
    uint32_t n_tensors;
    float max_norm, lr;
    float *norm;
    double *work;        // clip_sums()
};
// A tensor is read in chunks of 4096 elements.  A job's tensors go in groups of kClipTensors, and a group has a sum of squares for each of its workgroups: one per
// chunk, but no more than kClipSums.  clip_sums: those of a job, whose tensor i has count(i) elements.
constexpr uint32_t kClipChunkBits = 12, kClipSums = 1024, kClipTensors = 64;
inline uint64_t clip_chunks(uint64_t count) { return (count + (1ull << kClipChunkBits) - 1) >> kClipChunkBits; }
template <typename Count>
inline uint64_t clip_sums(uint32_t n, Count count)
{
    uint64_t sums = 0;
    for (uint32_t i = 0; i < n; i += kClipTensors) {
        uint64_t chunks = 0;
        for (uint32_t k = i; k < n && k < i + kClipTensors; ++k) chunks += clip_chunks(count(k));
        sums += chunks < kClipSums ? chunks : kClipSums;
    }
    return sums;
}
hipError_t launch_clip(const ClipJob *jobs, uint32_t n, bool sgd, hipStream_t stream, uint64_t *launches);

}  // namespace salus
