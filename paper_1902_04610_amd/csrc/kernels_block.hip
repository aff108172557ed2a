// Products of transformer blocks, all jobs of a round in one launch: the two of a gated feed-forward block, Y = (act(X Wg) * (X Wu))
// Wout + R, a dense layer act(X W + b) + R, and the input gradients of both.  What follows a product (bias, activation,
// the product of the halves, the residual, the gate's derivative) happens on its float sums on the way to memory (block.hpp), so that
// a round of dense layers is one launch and one of gated blocks is two.
#include <algorithm>

#include "block_launch.hpp"
#include "narrow_tile.hpp"

namespace salus {

// Few rows (at most 16 MT): tiles of 16 NB columns of weights, K split over the four wavefronts of a workgroup, weights straight into an LDS ring per
// wavefront (NarrowTile).  Gated: half the columns are the gate's.  TWO: two workgroups per compute unit.
template <int MT, int NB, bool TWO, bool GATED, typename Args>
__device__ inline void narrow_block(const Args &a, unsigned char *smem)
{
    using T = std::conditional_t<TWO, NarrowTile<MT, NB, 1, 80 * 1024>, NarrowTile<MT, NB>>;
    constexpr uint32_t kCols = GATED ? 8 * NB : 16 * NB;
    BlockProblem p;
    const uint32_t t = find_owner(a.first, a.p, xcd_remap(blockIdx.x + a.base, a.tiles), p);
    const uint32_t M = p.M, N = p.N, act = p.flags & 0xffu, rt = (M + 16 * MT - 1) / (16 * MT);
    const Tile tile = {t % rt * 16 * MT, t / rt * kCols};      // row tiles of one column tile are neighbours: they share W
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto row_of = [&](int i) { return tile.m0 + 16u * i + 4u * g + wave; };
    float own[MT * NB];
    if constexpr (GATED) {
        T::template sums<true, true>(p.W, p.X, M, p.K, N, false, false, N * 4u, N * 2u, tile, smem, own);
        constexpr int H = NB / 2;
        float h[MT * H];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) {
                const uint32_t row = row_of(i), n = tile.n0 + 16 * j + c;
                const float gate = own[i * NB + j];
                if (p.Z && row < M && n < N) {
                    Global<float> *Z = (Global<float> *)p.Z + (size_t)row * (2 * N) + n;
                    Z[0] = gate;
                    Z[N] = own[i * NB + H + j];
                }
                h[i * H + j] = gate;
            }
        activate_all(h, act, false);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) {
                const uint32_t row = row_of(i), n = tile.n0 + 16 * j + c;
                if (row < M && n < N) ((Global<uint16_t> *)p.Y)[(size_t)row * N + n] = (uint16_t)bf16_bits(h[i * H + j] * own[i * NB + H + j]);
            }
    } else {
        // bias and residual are asked for in front of everything else
        uint16_t r[MT * NB] = {}, b[NB] = {};
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const uint32_t n = tile.n0 + 16 * j + c;
            if (p.B && n < N) b[j] = ((const Global<uint16_t> *)p.B)[n];
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (p.R && row_of(i) < M && n < N) r[i * NB + j] = ((const Global<uint16_t> *)p.R)[(size_t)row_of(i) * N + n];
        }
        T::template sums<false, true>(p.W, p.X, M, p.K, N, false, false, N * 2u, 0, tile, smem, own);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const uint32_t row = row_of(i), n = tile.n0 + 16 * j + c;
                own[i * NB + j] += bf16_low(b[j]);
                if (p.Z && row < M && n < N) ((Global<float> *)p.Z)[(size_t)row * N + n] = own[i * NB + j];
            }
        const bool out_bf16 = (p.flags & kOutBf16) != 0;
        activate_all(own, act, !out_bf16);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const uint32_t row = row_of(i), n = tile.n0 + 16 * j + c;
                if (row >= M || n >= N) continue;
                const float v = own[i * NB + j] + bf16_low(r[i * NB + j]);
                if (out_bf16) ((Global<uint16_t> *)p.Y)[(size_t)row * N + n] = (uint16_t)bf16_bits(v);
                else ((Global<float> *)p.Y)[(size_t)row * N + n] = v;
            }
    }
}
template <int MT, int NB, bool TWO, bool GATED, typename Args>
__global__ __launch_bounds__(kGemmThreads, TWO ? 2 : 1) void block_narrow(Args a)
{
    using T = std::conditional_t<TWO, NarrowTile<MT, NB, 1, 80 * 1024>, NarrowTile<MT, NB>>;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[T::kLds];
    narrow_block<MT, NB, TWO, GATED>(a, smem);
}

// The gate's derivative for few rows or few tiles: 16 CPL columns, K split over the four wavefronts, weights through registers, whose lanes load 16 bytes along
// a transposed weight's rows as it is (dense_bf16_sums).  Deep layers keep eight or four k-steps in flight instead of two.
template <int MT, int CPL, int D>
__device__ inline void narrow_gate_grad(const BlockProblem &p, const Tile tile, float *lds)
{
    float own[MT * CPL];
    dense_bf16_sums<MT, true, false, CPL, D>(p, tile, lds, own);
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t N = p.N, n = tile.n0 + CPL * c;
    typedef float vec __attribute__((ext_vector_type(CPL)));
    typedef uint32_t out_vec __attribute__((ext_vector_type(CPL / 2)));
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const uint32_t row = tile.m0 + 16 * t + 4 * g + wave;
        if (row >= p.M || n >= N) continue;
        const Global<float> *Z = (const Global<float> *)p.Z + (size_t)row * (2 * N) + n;
        const vec gate = *(const Global<vec> *)Z, up = *(const Global<vec> *)(Z + N);
        float z[CPL], du[CPL], dg[CPL];
#pragma unroll
        for (int i = 0; i < CPL; ++i) z[i] = gate[i];
        activate_with_slope(z, du, dg, p.flags & 0xffu);
        out_vec og, ou;
#pragma unroll
        for (int i = 0; i < CPL; i += 2) {
            og[i / 2] = bf16_pack(own[t * CPL + i] * up[i] * dg[i], own[t * CPL + i + 1] * up[i + 1] * dg[i + 1]);
            ou[i / 2] = bf16_pack(own[t * CPL + i] * du[i], own[t * CPL + i + 1] * du[i + 1]);
        }
        Global<uint16_t> *Y = (Global<uint16_t> *)p.Y + (size_t)row * (2 * N) + n;
        *(Global<out_vec> *)Y = og;
        *(Global<out_vec> *)(Y + N) = ou;
    }
}
constexpr uint32_t kGateDeepK = 2048;
template <int MT, int CPL, typename Args>
__global__ __launch_bounds__(kGemmThreads) void block_gate_grad_narrow(Args a)
{
    __shared__ float lds[reduce_lds_floats<MT * CPL>()];
    BlockProblem p;
    const uint32_t t = find_owner(a.first, a.p, xcd_remap(blockIdx.x + a.base, a.tiles), p), rt = (p.M + 16 * MT - 1) / (16 * MT);
    const Tile tile = {t % rt * 16 * MT, t / rt * 16 * CPL};
    if (p.K > kGateDeepK) narrow_gate_grad<MT, CPL, 16 / CPL>(p, tile, lds);
    else narrow_gate_grad<MT, CPL, 2>(p, tile, lds);
}

template <int MT, int NB, bool TWO, Epilogue E>
static hipError_t narrow(const Round &r)
{
    constexpr bool kGated = E == Epilogue::kGated;
    constexpr uint32_t kCols = kGated ? 8 * NB : 16 * NB;
    if (r.n <= kBlockFew)
        return launch_block<BlockFewArgs>(block_narrow<MT, NB, TWO, kGated, BlockFewArgs>, kGemmThreads, 16 * MT, kCols, 0, r.p, r.n, r.stream, r.launches);
    return launch_block<BlockArgs>(block_narrow<MT, NB, TWO, kGated, BlockArgs>, kGemmThreads, 16 * MT, kCols, 0, r.p, r.n, r.stream, r.launches);
}
template <int MT, int CPL>
static hipError_t narrow_grad(const Round &r)
{
    if (r.n <= kBlockFew)
        return launch_block<BlockFewArgs>(block_gate_grad_narrow<MT, CPL, BlockFewArgs>, kGemmThreads, 16 * MT, 16 * CPL, 0, r.p, r.n, r.stream, r.launches);
    return launch_block<BlockArgs>(block_gate_grad_narrow<MT, CPL, BlockArgs>, kGemmThreads, 16 * MT, 16 * CPL, 0, r.p, r.n, r.stream, r.launches);
}
// The times are fitted to launches of drawn sizes: 1 - 48 jobs of 1 - 4096 rows, widths of 64 - 8192; 210 dense, 105 gated, 61 gate gradients, 100 input
// gradients, kernel traces of every kind of tile on each of them; off by 6 - 10 % in the median.  The choice is 1.9 % (dense), 2.7 % (gated) and
// 1.9 % (gate gradients) off the quickest kind on average and 28, 33 and 34 % at most; the best single kind is 38 (64 x 64), 32 (64 x 128) and
// 25 % (32 x 32) off.
// What each is for: narrow tiles fill the chip with few rows, the ring streams weights past one or two row tiles, large tiles multiply.
//   1 job x 1 row, 4096 -> 1024: 16 columns 9.4 us, the ring 16
//   32 jobs x 1 - 32 rows, 1000 -> 5520: 64 x 64 75 us, 128 x 128 73, 128 x 256 73; 2760 -> 1000: 37, 37, 55
//   8 jobs x 64 rows, 2736 -> 1024: 32 x 64 20.7 us, 64 x 64 25.8
//   8 jobs x 1000 rows, 2048 -> 8192: 64 x 128 545 us, 128 x 128 353, 128 x 256 295, 256 x 256 286
// The 64 x 64 ring has three workgroups of three stages on a compute unit and is listed with two, as what it was fitted with, two of four stages: it takes
// 0.99 of their time over 27 drawn launches (0.90 - 1.0 above 512 tiles), which is how its numbers were scaled.
// One 128 x 128 tile per compute unit: eight wavefronts instead of four, 4 jobs x 500 rows, 2048 -> 2048, 27.5 / 29.2 us, 2 x 2000, 1024 -> 1024,
// 18.3 / 19.7, 0.95 over 10 drawn launches of 130 - 256 tiles (gated and gate gradients: 0.98 - 1.04, not there); its time is set as the same
// share of the other's.
constexpr Tiling kDense[] = {
    {16, 16, 1, 0, 16, 1300, 92, 1370, narrow<1, 1, false, Epilogue::kDense>},
    {32, 16, 1, 16, kAnyRows, 1300, 152, 1480, narrow<2, 1, false, Epilogue::kDense>},
    {16, 32, 1, 0, 16, 1100, 109, 1870, narrow<1, 2, false, Epilogue::kDense>},
    {32, 32, 1, 16, kAnyRows, 1100, 178, 2140, narrow<2, 2, false, Epilogue::kDense>},
    {16, 64, 2, 0, 16, 1400, 243, 3080, narrow<1, 4, true, Epilogue::kDense>},
    {32, 64, 2, 16, kAnyRows, 1800, 378, 3280, narrow<2, 4, true, Epilogue::kDense>},
    {64, 64, 2, 0, kAnyRows, 2400, 466, 2490, ring<64, 64, 2, 2, 3, 3, Epilogue::kDense>},
    {128, 128, 2, 0, kAnyRows, 2900, 923, 6250, tiled<128, 128, 2, 2, 2, Epilogue::kDense>},
    {128, 128, 1, 0, kAnyRows, 2800, 532, 3600, tiled<128, 128, 2, 4, 1, Epilogue::kDense>},
    {128, 256, 2, 0, kAnyRows, 2900, 1439, 10780, tiled<128, 256, 1, 4, 2, Epilogue::kDense>},
    {128, 256, 2, 0, 128, 2900, 1340, 10000, tiled<128, 256, 1, 4, 2, Epilogue::kDense, true>, true},
    {256, 256, 1, 0, kAnyRows, 0, 1180, 11130, tiled<256, 256, 2, 4, 1, Epilogue::kDense>},
};
constexpr Tiling kGated[] = {      // half of a tile's columns are the gate's
    {16, 16, 1, 0, 16, 1100, 166, 1560, narrow<1, 2, false, Epilogue::kGated>},
    {32, 16, 1, 16, kAnyRows, 1700, 248, 1110, narrow<2, 2, false, Epilogue::kGated>},
    {16, 32, 2, 0, 16, 1400, 341, 2450, narrow<1, 4, true, Epilogue::kGated>},
    {32, 32, 2, 16, kAnyRows, 2300, 499, 1040, narrow<2, 4, true, Epilogue::kGated>},
    {64, 64, 2, 0, kAnyRows, 2400, 806, 2280, ring<64, 128, 2, 2, 3, 2, Epilogue::kGated>},
    {128, 64, 2, 0, kAnyRows, 2400, 1036, 3920, tiled<128, 128, 2, 2, 2, Epilogue::kGated>},
    {128, 128, 2, 0, kAnyRows, 1400, 1471, 8870, tiled<128, 256, 1, 4, 2, Epilogue::kGated>},
    {128, 128, 2, 0, 128, 1400, 1370, 8300, tiled<128, 256, 1, 4, 2, Epilogue::kGated, true>, true},
    {256, 128, 1, 0, kAnyRows, 800, 1259, 8090, tiled<256, 256, 2, 4, 1, Epilogue::kGated>},
};
constexpr Tiling kGateGrad[] = {
    {16, 32, 1, 0, 16, 2800, 121, 230, narrow_grad<1, 2>},
    {32, 32, 1, 16, kAnyRows, 2500, 165, 830, narrow_grad<2, 2>},
    {16, 64, 1, 0, 16, 3000, 209, 270, narrow_grad<1, 4>},
    {32, 64, 1, 16, kAnyRows, 2700, 269, 1120, narrow_grad<2, 4>},
    {64, 64, 2, 0, kAnyRows, 2000, 442, 4720, ring<64, 64, 2, 2, 3, 3, Epilogue::kGateGrad>},
    {64, 128, 2, 0, kAnyRows, 800, 627, 8500, ring<64, 128, 2, 2, 3, 2, Epilogue::kGateGrad>},
    {128, 128, 2, 0, kAnyRows, 0, 904, 14890, tiled<128, 128, 2, 2, 2, Epilogue::kGateGrad>},
    {256, 256, 1, 0, kAnyRows, 0, 1074, 19050, tiled<256, 256, 2, 4, 1, Epilogue::kGateGrad>},
};
hipError_t launch_block_dense(const BlockProblem *p, uint32_t n, bool cached, hipStream_t stream, uint64_t *launches)
{
    return choose(kDense, p, n, cached).tiling->launch({p, n, stream, launches});
}

hipError_t launch_block_gated(const BlockProblem *p, uint32_t n, bool cached, hipStream_t stream, uint64_t *launches)
{
    return choose(kGated, p, n, cached, 4).tiling->launch({p, n, stream, launches});
}

hipError_t launch_block_gate_grad(const BlockProblem *p, uint32_t n, bool cached, hipStream_t stream, uint64_t *launches)
{
    return choose(kGateGrad, p, n, cached).tiling->launch({p, n, stream, launches});
}

// ---- slope of a dense layer -----------------------------------------------------------------------------------------------------
// dZ = dY * act'(Z), rounded to bf16 as a factor of dX and dW, and the column sums of dZ before its rounding.  A workgroup takes 16 rows of 512 columns, a wavefront four of the rows, a lane
// eight columns; all of a lane's loads are on their way together.  The four wavefronts' sums are added in the order of the rows.  Bound by memory:
// 8 bytes an element (2 and 4 read, 2 written).
struct SlopeArgs {
    uint32_t n, tiles, base, pad;
    uint32_t first[kBlockProblems];
    SlopeProblem p[kBlockProblems];
};
static_assert(sizeof(SlopeArgs) <= 4096, "kernel arguments are limited to 4 KB");
constexpr uint32_t kSlopeCols = 512, kSlopeWaveRows = kSlopeRows / kWaves;

__global__ __launch_bounds__(64 * kWaves) void block_slope(SlopeArgs a)
{
    __shared__ float part[kWaves][8][64];
    SlopeProblem p;
    const uint32_t t = find_owner(a.first, a.p, blockIdx.x + a.base, p), ct = (p.N + kSlopeCols - 1) / kSlopeCols;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t block = t / ct, row0 = block * kSlopeRows + wave * kSlopeWaveRows, c = (t % ct) * kSlopeCols + 8 * lane;
    const bool in = c < p.N;
    const Global<uint16_t> *dY = (const Global<uint16_t> *)p.dY + (in ? c : 0);
    const Global<float> *Z = (const Global<float> *)p.Z + (in ? c : 0);
    u32x4 w[kSlopeWaveRows];
    f32x4 z[kSlopeWaveRows][2];
#pragma unroll
    for (uint32_t r = 0; r < kSlopeWaveRows; ++r) {
        const size_t at = (size_t)min(row0 + r, p.M - 1) * p.N;      // rows past the last: read again, not used
        w[r] = *(const Global<u32x4> *)(dY + at);
        if (!p.Z) continue;
        z[r][0] = *(const Global<f32x4> *)(Z + at);
        z[r][1] = *(const Global<f32x4> *)(Z + at + 4);
    }
    float sum[8] = {};
#pragma unroll
    for (uint32_t r = 0; r < kSlopeWaveRows; ++r) {
        if (row0 + r >= p.M) break;
        float v[8], slope[8], unused[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = e & 1 ? bf16_high(w[r][e / 2]) : bf16_low(w[r][e / 2]);
            slope[e] = z[r][e / 4][e & 3];
        }
        if (p.Z) {
            float at[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) at[e] = slope[e];
            activate_with_slope(at, unused, slope, p.act);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= slope[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
        if (p.dZ && in)
            *(Global<u32x4> *)((Global<uint16_t> *)p.dZ + (size_t)(row0 + r) * p.N + c) =
                u32x4{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7])};
    }
    if (!p.db) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) part[wave][e][lane] = sum[e];
    __syncthreads();
    // thread: two of the 512 columns, which lie at [wave][column % 8][column / 8]
    Global<float> *to = (Global<float> *)(p.M <= kSlopeRows ? p.db : p.partial + (size_t)block * p.N);
#pragma unroll
    for (uint32_t i = 0; i < kSlopeCols / 256; ++i) {
        const uint32_t column = 256 * i + threadIdx.x, n = (t % ct) * kSlopeCols + column;
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < kWaves; ++q) s += part[q][column & 7][column >> 3];
        if (n < p.N) to[n] = s;
    }
}

hipError_t launch_block_slope(const SlopeProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    for (uint32_t at = 0; at < n; at += kBlockProblems) {
        const uint32_t count = std::min(kBlockProblems, n - at);
        SlopeArgs a{};
        const uint64_t tiles = fill_group(a, p + at, count, [](const SlopeProblem &q) {
            return q.dZ || q.db ? (uint64_t)((q.M + kSlopeRows - 1) / kSlopeRows) * ((q.N + kSlopeCols - 1) / kSlopeCols) : 0;
        });
        if (tiles > 0x7fffffffull) return hipErrorInvalidValue;
        const hipError_t e = launch_tiles(tiles, launches, [&](uint32_t blocks, uint32_t base) {
            a.base = base;
            hipLaunchKernelGGL(block_slope, dim3(blocks), dim3(256), 0, stream, a);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace salus
