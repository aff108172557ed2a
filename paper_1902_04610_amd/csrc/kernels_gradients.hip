// What a backward pass of transformer blocks ends with: input gradients dX = G . W^T, weight gradients dW = X^T . G (bf16 out of float sums) and a dense
// layer's bias gradients, of all jobs and weights of a round.  None waits for another, and where each would leave compute units or their pipes idle, they
// share a launch.
#include <algorithm>
#include <vector>

#include "block_launch.hpp"

namespace salus {

template <typename P, uint32_t PROBLEMS>
struct Problems {
    uint32_t n, tiles, pad[2];
    uint32_t first[PROBLEMS];      // first tile of problem i; kNoTile from n on
    P p[PROBLEMS];
};
typedef Problems<WeightGradProblem, 64> WeightGradArgs;
typedef Problems<SlopeProblem, 32> SumArgs;
static_assert(sizeof(WeightGradArgs) <= 4096 && sizeof(SumArgs) <= 4096, "kernel arguments are limited to 4 KB");

// A launch of all three kinds: workgroups [0, sums) add columns, the next `inputs` walk the tiles of input gradients, the others take weight gradients.
constexpr uint32_t kSharedJobs = 16;
struct SharedArgs {
    uint32_t sums, inputs, weights, pad;
    Problems<BlockProblem, kSharedJobs> input;
    Problems<WeightGradProblem, 2 * kSharedJobs> weight;
    Problems<SlopeProblem, kSharedJobs> sum;
};
static_assert(sizeof(SharedArgs) <= 4096, "kernel arguments are limited to 4 KB");

// Both operands lie with their rows along the contraction and are transposed on the way out of LDS.  M side: X (rows of dW), N side: G.
template <int BM, int BN, typename Args = WeightGradArgs>
struct WeightGradWalk {
    static constexpr uint32_t kProblems = sizeof(Args::first) / 4;
    const Args &a;
    const uint32_t first;      // lane i: the first tile of problem i
    struct Place { int problem; uint32_t m0, n0, depth; };
    __device__ explicit WeightGradWalk(const Args &args) : a(args), first(args.first[min(threadIdx.x & 63, kProblems - 1)]) {}
    __device__ uint32_t tiles() const { return a.tiles; }
    __device__ Place place(uint32_t tile_id) const
    {
        const uint32_t id = xcd_remap(tile_id, a.tiles);
        const int g = __builtin_amdgcn_readfirstlane(wave_find_range(first, id, (threadIdx.x & 63) < kProblems));
        const WeightGradProblem &p = a.p[g];
        const uint32_t t = id - __builtin_amdgcn_readlane(first, g), rt = (p.K + BM - 1) / BM, ct = (p.N + BN - 1) / BN;
        const uint32_t band = t / (8u * ct), local = t - band * 8u * ct, rows = min(8u, rt - band * 8u);
        return {g, (band * 8u + local % rows) * BM, (local / rows) * BN, p.M};
    }
    __device__ Operand m(const Place &at) const { const WeightGradProblem &p = a.p[at.problem]; return {p.X, p.M, p.K, p.K * 2u, false}; }
    __device__ Operand n(const Place &at) const { const WeightGradProblem &p = a.p[at.problem]; return {p.G, p.M, p.N, p.N * 2u, false}; }
    struct Held {};
    __device__ void begin(const Place &, Held &, uint32_t, uint32_t, int) const {}
    template <int FN, int FM, typename Landed>
    __device__ void finish(const Place &place, const f32x16 (&acc)[FN][FM], const Held &, uint32_t m, uint32_t n, int lane, Landed landed) const
    {
        static_assert(FN % 2 == 0, "two blocks are stored together");
        const WeightGradProblem &p = a.p[place.problem];
        m += place.m0;
        n += place.n0;
        const uint32_t rows = m < p.K ? p.K - m : 0, cols = n < p.N ? p.N - n : 0, column = line_column_bf16(lane);
        uint16_t *dW = (uint16_t *)p.dW + (uint64_t)m * p.N + n;
        landed();
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; j += 2) {
                __builtin_amdgcn_sched_barrier(0);
                float v[2][16];
#pragma unroll
                for (int jj = 0; jj < 2; ++jj)
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[jj][r] = acc[j + jj][i][r];
                u32x4 o[2][2];
                to_lines_bf16(v, o);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t r = 32u * i + 8u * q + (lane & 7), c = 32u * j + column;
                    if (r < rows && c < cols) *(u32x4 *)(dW + (size_t)r * p.N + c) = o[q >> 1][q & 1];
                }
            }
    }
};

template <int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void weight_grad_tiled(WeightGradArgs a)
{
    using T = TileMfma<BM, BN, WM, WN, true, true>;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[T::kLds];
    const WeightGradWalk<BM, BN> walk(a);
    T::run(walk, smem);
}

// Few rows: what bounds it is the writing of dW.  A wavefront owns 64 x 64 of dW, a workgroup four such blocks side by side.  Lane (c, g) loads the 8 x 4
// blocks X[m + 8g ..][k0 + 4c ..] and G[m + 8g ..][n0 + 4c ..] of a step of 32 rows, transposes them in registers into four A and four B operands
// of v_mfma_f32_16x16x32_bf16, and ends up with 16 rows x 4 consecutive columns: 128 contiguous bytes per row across the 16 lanes.  What is
// wanted of up to 64 rows is asked for at once.
// An XCD has a run of blocks down the rows of dW, which share their columns of G and, job by job, X in its L2, and three workgroups per compute unit:
// 8 jobs x 64 rows, 1024 -> 5472 and 2736 -> 1024 (134 MB of dW), 33.9 us, with blocks along the rows of dW dealt round-robin to the XCDs 43.9.
// Four blocks below each other by one workgroup, G kept in registers: 31.7, but 1.4 of the time on average over 25 launches of 1 - 96 rows.
constexpr uint32_t kFewBlock = 64, kFewCols = 256, kFewSteps = 2;
template <typename Args>
__device__ inline void few_rows(const Args &a, uint32_t id)
{
    WeightGradProblem p;
    const uint32_t t = find_owner(a.first, a.p, xcd_remap(id, a.tiles), p);
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t M = p.M, K = p.K, N = p.N, kt = (K + kFewBlock - 1) / kFewBlock;
    const uint32_t k0 = t % kt * kFewBlock, n0 = t / kt * kFewCols + kFewBlock * wave;
    if (n0 >= N) return;
    const uint32_t kcol = k0 + 4 * c, ncol = n0 + 4 * c;
    // rows and columns outside the matrices: a valid address, and what comes of it is not stored or, past the last row, dropped
    const Global<uint16_t> *X = (const Global<uint16_t> *)p.X + (kcol < K ? kcol : 0);
    const Global<uint16_t> *G = (const Global<uint16_t> *)p.G + (ncol < N ? ncol : 0);
    f32x4 acc[16];      // [i * 4 + j][r]
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x2 h[kFewSteps][8], d[kFewSteps][8];
    auto load = [&](int s, uint32_t m0) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const size_t m = min(m0 + 8 * g + r, M - 1);
            h[s][r] = *(const Global<u32x2> *)(X + m * K);
            d[s][r] = *(const Global<u32x2> *)(G + m * N);
        }
    };
    auto multiply = [&](int s, uint32_t m0) {
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (m0 + 8 * g + r >= M) {
                h[s][r] = u32x2{0u, 0u};
                d[s][r] = u32x2{0u, 0u};
            }
        u32x4 A[4], B[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t sel = (i & 1) ? 0x07060302u : 0x05040100u;
                A[i][j] = __builtin_amdgcn_perm(h[s][2 * j + 1][i >> 1], h[s][2 * j][i >> 1], sel);
                B[i][j] = __builtin_amdgcn_perm(d[s][2 * j + 1][i >> 1], d[s][2 * j][i >> 1], sel);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i * 4 + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, A[i]), __builtin_bit_cast(bf16x8, B[j]), acc[i * 4 + j], 0, 0, 0);
    };
    for (uint32_t m0 = 0; m0 < M; m0 += 32 * kFewSteps) {
#pragma unroll
        for (int s = 0; s < (int)kFewSteps; ++s)
            if (m0 + 32u * s < M) load(s, m0 + 32u * s);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < (int)kFewSteps; ++s)
            if (m0 + 32u * s < M) multiply(s, m0 + 32u * s);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t krow = k0 + 16 * g + 4 * r + i;
            if (krow < K && ncol < N)
                *(Global<u32x2> *)((Global<uint16_t> *)p.dW + (size_t)krow * N + ncol) =
                    u32x2{bf16_pack(acc[4 * i][r], acc[4 * i + 1][r]), bf16_pack(acc[4 * i + 2][r], acc[4 * i + 3][r])};
        }
}

__global__ __launch_bounds__(256, 3) void weight_grad_few_rows(WeightGradArgs a) { few_rows(a, blockIdx.x); }

// db of jobs of more than 16 rows: the blocks' sums.  A workgroup takes 64 columns, 16 threads four of them each, and thread group g the blocks g, g + 16, ..;
// the groups are added in order.
template <typename Args>
__device__ inline void column_sums(const Args &a, uint32_t id, float (*part)[64])
{
    SlopeProblem p;
    const uint32_t c0 = find_owner(a.first, a.p, id, p) * 64u, group = threadIdx.x >> 4, c = c0 + 4 * (threadIdx.x & 15);
    const uint32_t blocks = (p.M + kSlopeRows - 1) / kSlopeRows;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (c < p.N) {
#pragma unroll 4
        for (uint32_t b = group; b < blocks; b += 16) sum += *(const Global<f32x4> *)((const Global<float> *)p.partial + (size_t)b * p.N + c);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) part[group][4 * (threadIdx.x & 15) + e] = sum[e];
    __syncthreads();
    if (threadIdx.x >= 64 || c0 + threadIdx.x >= p.N) return;
    float s = 0.0f;
#pragma unroll
    for (int g = 0; g < 16; ++g) s += part[g][threadIdx.x];
    ((Global<float> *)p.db)[c0 + threadIdx.x] = s;
}

constexpr uint32_t kSumBytes = 16 * 64 * 4;
__global__ __launch_bounds__(256) void block_column_sums(SumArgs a)
{
    __shared__ float part[16][64];
    column_sums(a, blockIdx.x, part);
}

// All three in a launch.  Few rows: input gradients through the ring, of which few and long tiles leave most of the chip's bandwidth, and weight
// gradients, which write.  More: 128 x 128 tiles of both, two workgroups per compute unit, one of which multiplies while the other begins or ends.
__global__ __launch_bounds__(256, 3) void gradients_few_rows(SharedArgs a)
{
    using T = TileStream<64, 64, 2, 2, false, 3>;
    static_assert(T::kLds >= kSumBytes && 3 * T::kLds <= 160 * 1024, "three workgroups per compute unit");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[T::kLds];
    uint32_t id = blockIdx.x;
    if (id < a.sums) {
        if (id < a.sum.tiles) column_sums(a.sum, id, (float (*)[64])smem);
        return;
    }
    id -= a.sums;
    if (id < a.inputs) {
        const BlockWalk<64, 64, Epilogue::kPlainT, decltype(a.input)> walk(a.input);
        T::run(walk, smem, id, a.inputs);
        return;
    }
    few_rows(a.weight, id - a.inputs);
}

__global__ __launch_bounds__(256, 2) void gradients_tiled(SharedArgs a)
{
    using TX = TileRows<128, 128, 2, 2>;
    using TW = TileMfma<128, 128, 2, 2, true, true>;
    constexpr uint32_t kLds = TX::kLds > TW::kLds ? TX::kLds : TW::kLds;
    static_assert(kLds >= kSumBytes && 2 * kLds <= 160 * 1024, "two workgroups per compute unit");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kLds];
    uint32_t id = blockIdx.x;
    if (id < a.sums) {
        if (id < a.sum.tiles) column_sums(a.sum, id, (float (*)[64])smem);
        return;
    }
    id -= a.sums;
    if (id < a.inputs) {
        const BlockWalk<128, 128, Epilogue::kPlainT, decltype(a.input)> walk(a.input);
        TX::run(walk, smem, id, a.inputs);
        return;
    }
    const WeightGradWalk<128, 128, decltype(a.weight)> walk(a.weight);
    TW::run(walk, smem, id - a.inputs, a.weights);
}

template <int BM, int BN, int WM, int WN>
static hipError_t launch_tiled_grad(const WeightGradProblem *p, uint32_t n, uint32_t per_cu, hipStream_t stream, uint64_t *launches)
{
    for (uint32_t at = 0; at < n; at += 64) {
        WeightGradArgs a{};
        const uint64_t tiles = fill_group(a, p + at, std::min(64u, n - at), [](const WeightGradProblem &q) {
            return (uint64_t)((q.K + BM - 1) / BM) * ((q.N + BN - 1) / BN);
        });
        if (tiles == 0) continue;
        if (tiles > 0x7fffffffull) return hipErrorInvalidValue;
        hipLaunchKernelGGL((weight_grad_tiled<BM, BN, WM, WN>), dim3((uint32_t)std::min<uint64_t>(tiles, per_cu * resident_grid())), dim3(64 * WM * WN), 0, stream, a);
        if (launches) *launches += 1;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

static hipError_t launch_few_rows(const WeightGradProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    for (uint32_t at = 0; at < n; at += 64) {
        WeightGradArgs a{};
        const uint64_t tiles = fill_group(a, p + at, std::min(64u, n - at), [](const WeightGradProblem &q) {
            return (uint64_t)((q.K + kFewBlock - 1) / kFewBlock) * ((q.N + kFewCols - 1) / kFewCols);
        });
        if (tiles == 0) continue;
        if (tiles > 0x7fffffffull) return hipErrorInvalidValue;
        hipLaunchKernelGGL(weight_grad_few_rows, dim3((uint32_t)tiles), dim3(256), 0, stream, a);
        if (launches) *launches += 1;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// A launch of tiles of `side` x `side`, per_cu at a time on a compute unit, in nanoseconds (Tiling in kernels_block.hip says how).
struct WeightTiling { uint32_t side, per_cu, fixed, slab, rest; };
constexpr WeightTiling kWeight128 = {128, 2, 2400, 1062, 2380}, kWeight256 = {256, 1, 0, 1500, 7500};
static uint64_t tiled_ns(const WeightGradProblem *p, uint32_t n, const WeightTiling &t)
{
    const uint64_t side = t.side, per_cu = t.per_cu, fixed = t.fixed, slab = t.slab, rest = t.rest;
    uint64_t tiles = 0, work = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const uint64_t count = (uint64_t)((p[i].K + side - 1) / side) * ((p[i].N + side - 1) / side);
        tiles += count;
        work += count * ((uint64_t)std::max((p[i].M + kSlab - 1) / kSlab, kMinSlabs) * slab + rest);
    }
    if (tiles == 0) return 0;
    const uint64_t cus = resident_grid(), grid = cus * per_cu, last = tiles % grid;
    return fixed + (tiles / grid * 10 + (last == 0 ? 0 : per_cu == 1 || last > cus ? 10 : 6)) * (work / tiles) / 10;
}

// Input gradients: large tiles, if they are quicker than what the grouped dense layers have for transposed weights (launch_grouped_bf16), for which its
// narrow and ring tiles stand here.
constexpr Tiling kInputLarge[] = {
    {128, 128, 2, 0, kAnyRows, 1400, 886, 3750, tiled<128, 128, 2, 2, 2, Epilogue::kPlainT>},
    {256, 256, 1, 0, kAnyRows, 0, 1033, 6770, tiled<256, 256, 2, 4, 1, Epilogue::kPlainT>},
};
constexpr Tiling kInputOther[] = {
    {16, 32, 1, 0, 16, 2000, 165, 500, nullptr},
    {32, 32, 1, 16, kAnyRows, 2000, 200, 800, nullptr},
    {64, 64, 2, 0, kAnyRows, 2100, 405, 1920, nullptr},
    {64, 128, 2, 0, kAnyRows, 1400, 605, 2940, nullptr},
};

// Register blocks if a weight's rows, on average over the weights, are at most 96: 0.55 - 0.84 of the time of 128 x 128 tiles for up to 64 rows (32 launches
// of 0.1 - 140 MB of dW), 0.92 - 1.19 for 66 - 85, 1.2 - 2.3 above 126.  Else 128 x 128 tiles, two per compute unit, or 256 x 256 ones, whichever
// should be quicker: 2 jobs x 4096 rows, 4096 -> 22016 and 11008 -> 4096, 3.09 and 1.92 ms, 4 jobs x 500, 2048 -> 2048, 24.5 / 23.0 us.  (Over 100
// launches of 1 - 4096 rows the choice between these two is 0.6 % off the quicker one.)
constexpr double kFewRows = 96;

static bool rows_are_few(const WeightGradProblem *p, uint32_t n)
{
    double rows = 0, weights = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const double w = (double)p[i].K * p[i].N;
        weights += w;
        rows += w * p[i].M;
    }
    return rows <= kFewRows * weights;
}

static hipError_t launch_weight_grad(const WeightGradProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    if (rows_are_few(p, n)) return launch_few_rows(p, n, stream, launches);
    if (tiled_ns(p, n, kWeight256) < tiled_ns(p, n, kWeight128)) return launch_tiled_grad<256, 256, 2, 4>(p, n, 1, stream, launches);
    return launch_tiled_grad<128, 128, 2, 2>(p, n, 2, stream, launches);
}

static hipError_t launch_input_grad(const BlockProblem *p, uint32_t n, bool cached, hipStream_t stream, uint64_t *launches)
{
    if (n == 0) return hipSuccess;
    const Choice large = choose(kInputLarge, p, n, true);
    if (large.ns < choose(kInputOther, p, n, true).ns) return large.tiling->launch({p, n, stream, launches});
    std::vector<Problem> q;
    q.reserve(n);
    for (uint32_t i = 0; i < n; ++i) q.push_back({p[i].W, p[i].X, p[i].Y, nullptr, p[i].M, p[i].K, p[i].N, kOutBf16});
    return launch_grouped_bf16(q.data(), n, true, cached, stream, launches);
}

static uint64_t sum_tiles(const SlopeProblem &q) { return (uint64_t)(q.N + 63) / 64; }

static hipError_t launch_sums(const SlopeProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    constexpr uint32_t kMost = sizeof(SumArgs::first) / 4;
    for (uint32_t at = 0; at < n; at += kMost) {
        SumArgs a{};
        const uint64_t tiles = fill_group(a, p + at, std::min(kMost, n - at), sum_tiles);
        hipLaunchKernelGGL(block_column_sums, dim3((uint32_t)tiles), dim3(256), 0, stream, a);
        if (launches) *launches += 1;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Tiles of 128 x 128 of a shared launch, two on a compute unit: how many, their times together and the longest, in nanoseconds.
struct SharedTiles { uint64_t tiles, work, longest; };
static SharedTiles shared_tiles(const BlockProblem *input, uint32_t n_input, const WeightGradProblem *weight, uint32_t n_weight)
{
    const Tiling &x = kInputLarge[0];
    SharedTiles s{};
    auto add = [&](uint64_t count, uint32_t depth, uint64_t slab, uint64_t rest) {
        const uint64_t ns = std::max((depth + kSlab - 1) / kSlab, kMinSlabs) * slab + rest;
        s.tiles += count;
        s.work += count * ns;
        s.longest = std::max(s.longest, ns);
    };
    for (uint32_t i = 0; i < n_input; ++i) add((uint64_t)((input[i].M + 127) / 128) * ((input[i].N + 127) / 128), input[i].K, x.slab, x.rest);
    for (uint32_t i = 0; i < n_weight; ++i) add((uint64_t)((weight[i].K + 127) / 128) * ((weight[i].N + 127) / 128), weight[i].M, kWeight128.slab, kWeight128.rest);
    return s;
}

// Do input and weight gradients share a launch of 128 x 128 tiles?  If its time is below that of the quickest launches of their own and 1.2 us for each
// launch that is saved (one that adds columns: 3.5).  Its time, from the tiles' as they run two on a compute unit: the longest tile, or all of them
// over all places and a quarter of the longest for the end; less a sixteenth, as they measured that much quicker than this says.
// Training calls of drawn sizes: 0.90 of the time where this shares; over 43 of them 0.97 if always shared, with 0.66 - 1.47 at the ends.
//   4 jobs x 500 rows, 2048 -> 2048: 43.9 us, alone 4.6 + 22.2 + 23.4
//   5 jobs x 125 - 262 rows, 704 -> 112: 18.9, alone 28.4
//   1 job x 486 rows, depth 14224, whose few input gradient tiles one compute unit walks alone: 197, alone 134
static bool share_tiled(const BlockProblem *input, uint32_t n_input, const WeightGradProblem *weight, uint32_t n_weight, bool sums)
{
    const SharedTiles s = shared_tiles(input, n_input, weight, n_weight);
    uint64_t longest = s.longest;
    const uint64_t cus = resident_grid();
    if (s.tiles <= cus) longest = longest * 6 / 10;
    const uint64_t shared = 2000 + std::max(longest, s.work / (2 * cus) + longest / 4);
    const uint64_t alone = std::min(choose(kInputLarge, input, n_input, true).ns, choose(kInputOther, input, n_input, true).ns) +
                           std::min(tiled_ns(weight, n_weight, kWeight128), tiled_ns(weight, n_weight, kWeight256));
    return shared - shared / 16 < alone + 1200 + (sums ? 3500 : 0);
}

// And a launch of ring tiles and register blocks?  Beside the writes an input gradient's tile takes up to twice as long: worth it unless that is what the
// launch lasts.  More than 16 rows: depth up to 4096, or any where dW is at most 64 MB; fewer, whose narrow tiles alone are quicker: depth up to
// 2048, or 4096 where there are half as many tiles as compute units.
// 83 training calls of drawn sizes, of which 45 are of few rows: 0.87 of the time on average where this shares.
//   7 jobs x 13 - 23 rows, depth 3232: 24.6 us, alone 2.8 + 11.7 + 11.8 + 14.7
//   3 jobs x 45 - 49 rows, 3696: 25.0, alone 17.9 + 14.9
//   2 jobs x 19 - 21 rows, 8032 (53 MB): 36.8, alone 29.2 + 13.3
//   8 jobs x 64 rows, 5472 (134 MB): 69, alone 25 + 34
//   1 job x 13 rows, 4256: 21.3, alone 12.5 + 6.0
static bool share_few_rows(const BlockProblem *input, uint32_t n_input, const WeightGradProblem *weight, uint32_t n_weight)
{
    uint64_t bytes = 0, tiles = 0;
    for (uint32_t i = 0; i < n_weight; ++i) bytes += 2ull * weight[i].K * weight[i].N;
    for (uint32_t i = 0; i < n_input; ++i) tiles += (uint64_t)((input[i].M + 63) / 64) * ((input[i].N + 63) / 64);
    const uint32_t many = bytes <= 64 << 20 ? ~0u : 4096u, few = tiles * 2 >= resident_grid() ? 4096u : 2048u;
    return std::all_of(input, input + n_input, [&](const BlockProblem &q) { return q.K <= (q.M > 16 ? many : few); });
}

hipError_t launch_gradients(const BlockProblem *input, uint32_t n_input, const WeightGradProblem *weight, uint32_t n_weight, const SlopeProblem *sums, uint32_t n_sums,
                            bool cached, hipStream_t stream, uint64_t *launches)
{
    const bool few = rows_are_few(weight, n_weight);
    if (n_input != 0 && n_input <= kSharedJobs && n_weight <= 2 * kSharedJobs && n_sums <= kSharedJobs &&
        (few ? share_few_rows(input, n_input, weight, n_weight) : share_tiled(input, n_input, weight, n_weight, n_sums != 0))) {
        SharedArgs a{};
        const uint32_t side = few ? 64 : 128;
        const uint64_t in = fill_group(a.input, input, n_input, [&](const BlockProblem &q) { return (uint64_t)((q.M + side - 1) / side) * ((q.N + side - 1) / side); });
        const uint64_t out = fill_group(a.weight, weight, n_weight, [&](const WeightGradProblem &q) {
            return few ? (uint64_t)((q.K + kFewBlock - 1) / kFewBlock) * ((q.N + kFewCols - 1) / kFewCols) : (uint64_t)((q.K + 127) / 128) * ((q.N + 127) / 128);
        });
        const uint64_t added = (fill_group(a.sum, sums, n_sums, sum_tiles) + 7) / 8 * 8;      // a multiple of 8: the others keep to their XCDs
        const uint64_t places = 2ull * resident_grid();
        if (in > 0x7fffffffull || out > 0x7fffffffull || added > 0x7fffffffull || in + out + added > 0x7fffffffull) return hipErrorInvalidValue;
        a.sums = (uint32_t)added;
        if (few) {
            a.inputs = (uint32_t)std::min(in, places);
            a.weights = (uint32_t)out;
            hipLaunchKernelGGL(gradients_few_rows, dim3(a.sums + a.inputs + a.weights), dim3(256), 0, stream, a);
        } else {
            // All of them have a place.  Else places (a multiple of 8 for the XCDs) go by the work, unless whole tiles fall much better otherwise: by
            // the time of the kind whose workgroups take longer and a quarter of the other's, a fifth less.
            //   4 jobs x 500 rows, 2048 -> 2048, 256 and 1024 tiles: 43.9 us on 256 and 256 places, 48.6 on 232 and 280
            //   10 x 400, 768 -> 768, 240 and 360 tiles: 21 / 23.4
            // Where the formula says less it is wrong as often as right: 9 jobs x 204 - 249 rows, 3280 -> 400, 14 % by the formula, 26.5 / 25.0;
            // 13 jobs x 490, 12 %, 793 / 845.
            uint64_t most = in;
            if (in + out > places) {
                // of a tile, two on a compute unit
                const uint64_t x = shared_tiles(input, n_input, nullptr, 0).work / in, y = shared_tiles(nullptr, 0, weight, n_weight).work / out;
                auto ns = [&](uint64_t i) {
                    const uint64_t i_ns = (in + i - 1) / i * x, w_ns = (out + places - i - 1) / (places - i) * y;
                    return std::max(i_ns, w_ns) + std::min(i_ns, w_ns) / 4;
                };
                const uint64_t all_x = launch_ns(kInputLarge[0], input, n_input), all_y = tiled_ns(weight, n_weight, kWeight128);
                const uint64_t by_work = std::min(places - 8, std::max<uint64_t>(8, places * all_x / (all_x + all_y) / 8 * 8));
                uint64_t whole = by_work;
                for (uint64_t i = 8; i < places; i += 8)
                    if (ns(i) < ns(whole)) whole = i;
                most = ns(whole) * 5 < ns(by_work) * 4 ? whole : by_work;
            }
            a.inputs = (uint32_t)std::min(in, most);
            a.weights = (uint32_t)std::min(out, places - a.inputs);
            hipLaunchKernelGGL(gradients_tiled, dim3(a.sums + a.inputs + a.weights), dim3(256), 0, stream, a);
        }
        if (launches) *launches += 1;
        return hipGetLastError();
    }
    hipError_t e = n_sums ? launch_sums(sums, n_sums, stream, launches) : hipSuccess;
    if (e == hipSuccess) e = launch_input_grad(input, n_input, cached, stream, launches);
    if (e == hipSuccess) e = launch_weight_grad(weight, n_weight, stream, launches);
    return e;
}

}  // namespace salus
