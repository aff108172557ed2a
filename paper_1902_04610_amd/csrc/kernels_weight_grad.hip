// Weight gradients of transformer blocks: dW = X^T . G, bf16 out of float sums, of all jobs and weights of a round in one launch.
#include <algorithm>

#include "block.hpp"

namespace salus {

struct WeightGradArgs {
    uint32_t n, tiles, pad[2];
    uint32_t first[64];
    WeightGradProblem p[64];
};
static_assert(sizeof(WeightGradArgs) <= 4096, "kernel arguments are limited to 4 KB");

// Both operands lie with their rows along the contraction and are transposed on the way out of LDS.  M side: X (rows of dW), N side: G.
template <int BM, int BN>
struct WeightGradWalk {
    const WeightGradArgs &a;
    const uint32_t first;      // lane i: the first tile of problem i
    struct Place { int problem; uint32_t m0, n0, depth; };
    __device__ explicit WeightGradWalk(const WeightGradArgs &args) : a(args), first(args.first[threadIdx.x & 63]) {}
    __device__ uint32_t tiles() const { return a.tiles; }
    __device__ Place place(uint32_t tile_id) const
    {
        const uint32_t id = xcd_remap(tile_id, a.tiles);
        const int g = __builtin_amdgcn_readfirstlane(wave_find_range(first, id, true));
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

// Few rows: what bounds it is the writing of dW.  A wavefront owns 64 x 64 of dW, a workgroup four such blocks side by side.  Lane (c, g) loads the 8 x 4 blocks X[m + 8g ..][k0 +
// 4c ..] and G[m + 8g ..][n0 + 4c ..] of a step of 32 rows, transposes them in registers into four A and four B operands of v_mfma_f32_16x16x32_bf16, and
// ends up with 16 rows x 4 consecutive columns: 128 contiguous bytes per row across the 16 lanes.  What is wanted of up to 64 rows is asked for at once.
constexpr uint32_t kFewBlock = 64, kFewCols = 256, kFewSteps = 2;
__global__ __launch_bounds__(256) void weight_grad_few_rows(WeightGradArgs a)
{
    WeightGradProblem p;
    const uint32_t t = find_owner(a.first, a.p, blockIdx.x, p);
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t M = p.M, K = p.K, N = p.N, nt = (N + kFewCols - 1) / kFewCols;
    const uint32_t k0 = t / nt * kFewBlock, n0 = t % nt * kFewCols + kFewBlock * wave;
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
static uint64_t tiled_ns(const WeightGradProblem *p, uint32_t n, uint32_t side, uint64_t per_cu, uint64_t fixed, uint64_t slab, uint64_t rest)
{
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

// Register blocks if a weight's rows, on average over the weights, are at most 96: 0.55 - 0.84 of the time of 128 x 128 tiles for up to 64 rows (32 launches of 0.1 - 140 MB of dW), 0.92 - 1.19 for 66 - 85,
// 1.2 - 2.3 above 126.  Else 128 x 128 tiles, two per compute unit, or 256 x 256 ones, whichever should be quicker: 2 jobs x 4096 rows, 4096 -> 22016 and 11008 -> 4096, 3.09 and 1.92 ms, 4 jobs x 500,
// 2048 -> 2048, 24.5 / 23.0 us.  (Over 100 launches of 1 - 4096 rows the choice between these two is 0.6 % off the quicker one.)
constexpr double kFewRows = 96;

hipError_t launch_weight_grad(const WeightGradProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    double rows = 0, weights = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const double w = (double)p[i].K * p[i].N;
        weights += w;
        rows += w * p[i].M;
    }
    if (rows <= kFewRows * weights) return launch_few_rows(p, n, stream, launches);
    if (tiled_ns(p, n, 256, 1, 0, 1282, 6660) < tiled_ns(p, n, 128, 2, 2400, 1062, 2380)) return launch_tiled_grad<256, 256, 2, 4>(p, n, 1, stream, launches);
    return launch_tiled_grad<128, 128, 2, 2>(p, n, 2, stream, launches);
}

}  // namespace salus
