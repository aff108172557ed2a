// Kernels on the tile walks of block.hpp, how they are launched, and the estimate that chooses between them.
#pragma once
#include <algorithm>
#include <type_traits>

#include "block.hpp"

namespace salus {

// 64-row tiles, operands through an LDS ring (TileStream), PER_CU workgroups per compute unit.  Right for every size: rows and columns outside
// are neither fetched nor stored.
template <int BM, int BN, int WM, int WN, int D, int PER_CU, Epilogue E>
__global__ __launch_bounds__(64 * WM * WN, WM * WN * PER_CU / 4) void block_stream(BlockArgs a)
{
    using Walk = BlockWalk<BM, BN, E>;
    using T = TileStream<BM, BN, WM, WN, !Walk::kTransposed, D, false, E == Epilogue::kGated>;
    static_assert(PER_CU * T::kLds <= 160 * 1024, "LDS of a compute unit");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[T::kLds];
    const Walk walk(a);
    T::run(walk, smem);
}

// Large tiles (TileMfma, TilePair, TileRows): where a weight is used by 128 rows and more, or comes in whole rounds of tiles.
// ONCE (128 x 256): weights that one row tile uses and that come from HBM are asked for non-temporally.
template <int BM, int BN, int WM, int WN, Epilogue E, bool ONCE = false>
__global__ __launch_bounds__(64 * WM * WN, 2) void block_tiled(BlockArgs a)
{
    using Walk = BlockWalk<BM, BN, E>;
    constexpr bool kPairs = E == Epilogue::kGated;
    using T = std::conditional_t<Walk::kTransposed, TileRows<BM, BN, WM, WN>,
                                 std::conditional_t<BM * BN == 128 * 256, TilePair<BM, BN, WM, WN, ONCE, kPairs>, TileMfma<BM, BN, WM, WN, false, true, kPairs>>>;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[T::kLds];
    const Walk walk(a);
    T::run(walk, smem);
}

// Launches of at most as many problems as Args holds: bm rows and `cols` output columns a tile, at most `grid` workgroups (0: one per tile).
template <typename Args>
inline hipError_t launch_block(void (*kernel)(Args), int threads, uint32_t bm, uint32_t cols, uint32_t grid, const BlockProblem *p, uint32_t n,
                               hipStream_t stream, uint64_t *launches)
{
    constexpr uint32_t kMost = sizeof(Args::first) / 4;
    for (uint32_t at = 0; at < n; at += kMost) {
        Args a{};
        const uint64_t tiles = fill_group(a, p + at, std::min(kMost, n - at),
                                          [&](const BlockProblem &q) { return (uint64_t)((q.M + bm - 1) / bm) * ((q.N + cols - 1) / cols); });
        if (tiles > 0x7fffffffull) return hipErrorInvalidValue;
        const hipError_t e = launch_tiles(grid ? std::min<uint64_t>(tiles, grid) : tiles, threads, launches, [&](uint32_t blocks, uint32_t base) {
            a.base = base;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, stream, a);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

struct Round {
    const BlockProblem *p;
    uint32_t n;
    hipStream_t stream;
    uint64_t *launches;
};

// One way to run a round: tiles of bm rows and `cols` columns of the output, per_cu of them at a time on a compute unit, for rounds whose largest job has
// more than `above` and at most `upto` rows; how long a launch takes in nanoseconds: fixed + rounds of tiles x (slabs of 64 of the depth x slab + rest).
struct Tiling {
    uint32_t bm, cols, per_cu, above, upto, fixed, slab, rest;
    hipError_t (*launch)(const Round &);
    bool once = false;       // asks for weights non-temporally: for weights from HBM and calls that do not need them again
};
// Bytes per nanosecond of weights from HBM: the most that tiles of fewer than 64 rows, other tiles, and tiles that ask non-temporally reached over the
// launches of more than 224 MB of weights.  32 jobs x 1 - 32 rows, gated 1000 -> 2760 and dense 2760 -> 1000 (530 MB): 128-row tiles
// non-temporal / cached 111 / 120 us.
// Whether weights come from HBM is a guess by what is resident in the pool (weights_cached), float masters and jobs without a turn among it.  Where
// it is wrong, weights that the cache holds beside 500 MB that no call touches, rounds take up to 1.15 of the time: 8 jobs x 128 rows,
// 1024 -> 2736 -> 1024, 36.8 / 42.0 us, 32 x 100, 512 -> 1024 -> 512, 29.8 / 33.1, 8 x 64, 1024 -> 2736 -> 1024, 32.7 / 32.7.
constexpr uint64_t kStreamNarrow = 4300, kStream = 4800, kStreamOnce = 5200;
constexpr uint32_t kAnyRows = ~0u;

inline uint64_t launch_ns(const Tiling &t, const BlockProblem *p, uint32_t n)
{
    uint64_t tiles = 0, work = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const uint64_t count = (uint64_t)((p[i].M + t.bm - 1) / t.bm) * ((p[i].N + t.cols - 1) / t.cols);
        tiles += count;
        work += count * ((uint64_t)std::max((p[i].K + kSlab - 1) / kSlab, kMinSlabs) * t.slab + t.rest);
    }
    if (tiles == 0) return 0;
    // a last round that leaves half of the compute units one tile instead of two takes 0.6 of the time of a full one
    const uint64_t cus = resident_grid(), grid = cus * t.per_cu, last = tiles % grid;
    const uint64_t tenths = tiles / grid * 10 + (last == 0 ? 0 : t.per_cu == 1 || last > cus ? 10 : 6);
    return t.fixed + tenths * (work / tiles) / 10;
}

struct Choice { const Tiling *tiling; uint64_t ns; };
// cached: as for launch_grouped_bf16; else no tiling is quicker than the weights' stream.  column_bytes: of a weight's row per output column.
template <size_t N>
inline Choice choose(const Tiling (&tilings)[N], const BlockProblem *p, uint32_t n, bool cached, uint32_t column_bytes = 2)
{
    uint32_t rows = 0;
    uint64_t bytes = 0;
    bool again = false;      // a backward pass, as what the forward pass leaves for it tells
    for (uint32_t i = 0; i < n; ++i) {
        rows = std::max(rows, p[i].M);
        bytes += (uint64_t)column_bytes * p[i].K * p[i].N;
        again = again || (p[i].flags & kReadAgain);
    }
    Choice best{nullptr, ~0ull};
    for (const Tiling &t : tilings) {
        if (rows <= t.above || rows > t.upto || (t.once && (cached || again))) continue;
        uint64_t ns = launch_ns(t, p, n);
        if (!cached) ns = std::max(ns, bytes / (t.once ? kStreamOnce : t.bm < 64 ? kStreamNarrow : kStream));
        if (ns < best.ns) best = {&t, ns};
    }
    return best;
}

template <int BM, int BN, int WM, int WN, int D, int PER_CU, Epilogue E>
inline hipError_t ring(const Round &r)
{
    return launch_block<BlockArgs>(block_stream<BM, BN, WM, WN, D, PER_CU, E>, 64 * WM * WN, BM, BlockWalk<BM, BN, E>::kCols, PER_CU * resident_grid(), r.p, r.n,
                                   r.stream, r.launches);
}
template <int BM, int BN, int WM, int WN, int PER_CU, Epilogue E, bool ONCE = false>
inline hipError_t tiled(const Round &r)
{
    return launch_block<BlockArgs>(block_tiled<BM, BN, WM, WN, E, ONCE>, 64 * WM * WN, BM, BlockWalk<BM, BN, E>::kCols, PER_CU * resident_grid(), r.p, r.n,
                                   r.stream, r.launches);
}

}  // namespace salus
