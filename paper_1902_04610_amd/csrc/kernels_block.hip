// Products of transformer blocks, all jobs of a round in one launch: the two of a gated feed-forward block, Y = (act(X Wg) * (X Wu))
// Wout + R, a dense layer act(X W + b) + R, and the input gradients of both.  What follows a product (bias, activation,
// the product of the halves, the residual, the gate's derivative) happens on its float sums on the way to memory (block.hpp), so that
// a round of dense layers is one launch and one of gated blocks is two.
#include <algorithm>

#include "block.hpp"

namespace salus {

// 64-row tiles, operands through an LDS ring (TileStream), two workgroups per compute unit.  Right for every size: rows and columns outside
// are neither fetched nor stored.
template <int BM, int BN, int WM, int WN, int D, Epilogue E>
__global__ __launch_bounds__(64 * WM * WN, 2) void block_stream(BlockArgs a)
{
    using Walk = BlockWalk<BM, BN, E>;
    using T = TileStream<BM, BN, WM, WN, !Walk::kTransposed, D, false, E == Epilogue::kGated>;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[T::kLds];
    const Walk walk(a);
    T::run(walk, smem);
}

template <int BM, int COLS>
static hipError_t launch_block(void (*kernel)(BlockArgs), int threads, uint32_t per_cu, const BlockProblem *p, uint32_t n, hipStream_t stream,
                               uint64_t *launches)
{
    for (uint32_t at = 0; at < n; at += kBlockProblems) {
        BlockArgs a{};
        const uint64_t tiles = fill_group(a, p + at, std::min(kBlockProblems, n - at),
                                          [](const BlockProblem &q) { return (uint64_t)((q.M + BM - 1) / BM) * ((q.N + COLS - 1) / COLS); });
        if (tiles == 0) continue;
        if (tiles > 0x7fffffffull) return hipErrorInvalidValue;
        const uint32_t grid = (uint32_t)std::min<uint64_t>(tiles, resident_grid() * per_cu);
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, stream, a);
        if (launches) *launches += 1;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_block_dense(const BlockProblem *p, uint32_t n, bool, hipStream_t stream, uint64_t *launches)
{
    return launch_block<64, 128>(block_stream<64, 128, 2, 2, 3, Epilogue::kDense>, 256, 2, p, n, stream, launches);
}

hipError_t launch_block_gated(const BlockProblem *p, uint32_t n, bool, hipStream_t stream, uint64_t *launches)
{
    return launch_block<64, 64>(block_stream<64, 128, 2, 2, 3, Epilogue::kGated>, 256, 2, p, n, stream, launches);
}

hipError_t launch_block_gate_grad(const BlockProblem *p, uint32_t n, bool, hipStream_t stream, uint64_t *launches)
{
    return launch_block<64, 128>(block_stream<64, 128, 2, 2, 3, Epilogue::kGateGrad>, 256, 2, p, n, stream, launches);
}

hipError_t launch_block_plain_t(const BlockProblem *p, uint32_t n, bool, hipStream_t stream, uint64_t *launches)
{
    return launch_block<64, 128>(block_stream<64, 128, 2, 2, 3, Epilogue::kPlainT>, 256, 2, p, n, stream, launches);
}

// ---- slope of a dense layer -----------------------------------------------------------------------------------------------------
// dZ = dY * act'(Z), and the column sums of dZ before its rounding: a workgroup takes 16 rows of 1024 columns, a thread four columns of
// them, one after the other, so that a sum's order is that of the rows.  Bound by memory: 8 bytes an element (2 and 4 read, 2 written).
struct SlopeArgs {
    uint32_t n, tiles, pad[2];
    uint32_t first[kBlockProblems];
    SlopeProblem p[kBlockProblems];
};
static_assert(sizeof(SlopeArgs) <= 4096, "kernel arguments are limited to 4 KB");
constexpr uint32_t kSlopeCols = 1024;

__global__ __launch_bounds__(256) void block_slope(SlopeArgs a)
{
    SlopeProblem p;
    const uint32_t t = find_owner(a.first, a.p, blockIdx.x, p), ct = (p.N + kSlopeCols - 1) / kSlopeCols;
    const uint32_t block = t / ct, row0 = block * kSlopeRows, c = (t % ct) * kSlopeCols + 4 * threadIdx.x;
    if (c >= p.N) return;
    const uint32_t rows = min(kSlopeRows, p.M - row0);
    const size_t corner = (size_t)row0 * p.N + c;
    const Global<uint16_t> *dY = (const Global<uint16_t> *)p.dY + corner;
    const Global<float> *Z = (const Global<float> *)p.Z + corner;
    Global<uint16_t> *dZ = (Global<uint16_t> *)p.dZ + corner;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t r = 0; r < rows; ++r) {
        const u32x2 w = *(const Global<u32x2> *)(dY + (size_t)r * p.N);
        float v[4] = {bf16_low(w[0]), bf16_high(w[0]), bf16_low(w[1]), bf16_high(w[1])};
        if (p.Z) {
            const f32x4 z = *(const Global<f32x4> *)(Z + (size_t)r * p.N);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= slope_fine(z[e], p.act);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[e];
        if (p.dZ) *(Global<u32x2> *)(dZ + (size_t)r * p.N) = u32x2{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3])};
    }
    if (!p.db) return;
    float *to = p.M <= kSlopeRows ? p.db : p.partial + (size_t)block * p.N;
    *(Global<f32x4> *)((Global<float> *)to + c) = sum;
}

// db of jobs of more than 16 rows: the blocks' sums, in row order.
__global__ __launch_bounds__(256) void block_column_sums(SlopeArgs a)
{
    SlopeProblem p;
    const uint32_t c = find_owner(a.first, a.p, blockIdx.x, p) * 256u + threadIdx.x;
    if (c >= p.N) return;
    const uint32_t blocks = (p.M + kSlopeRows - 1) / kSlopeRows;
    float sum = 0.0f;
    for (uint32_t b = 0; b < blocks; ++b) sum += ((const Global<float> *)p.partial)[(size_t)b * p.N + c];
    ((Global<float> *)p.db)[c] = sum;
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
        if (tiles) {
            hipLaunchKernelGGL(block_slope, dim3((uint32_t)tiles), dim3(256), 0, stream, a);
            if (launches) *launches += 1;
        }
        const uint64_t sums = fill_group(a, p + at, count, [](const SlopeProblem &q) { return q.db && q.M > kSlopeRows ? (uint64_t)(q.N + 255) / 256 : 0; });
        if (sums) {
            hipLaunchKernelGGL(block_column_sums, dim3((uint32_t)sums), dim3(256), 0, stream, a);
            if (launches) *launches += 1;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace salus
