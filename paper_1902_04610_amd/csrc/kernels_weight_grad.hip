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

hipError_t launch_weight_grad(const WeightGradProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    for (uint32_t at = 0; at < n; at += 64) {
        WeightGradArgs a{};
        const uint64_t tiles = fill_group(a, p + at, std::min(64u, n - at), [](const WeightGradProblem &q) {
            return (uint64_t)((q.K + 127) / 128) * ((q.N + 127) / 128);
        });
        if (tiles == 0) continue;
        if (tiles > 0x7fffffffull) return hipErrorInvalidValue;
        hipLaunchKernelGGL((weight_grad_tiled<128, 128, 2, 2>), dim3((uint32_t)std::min<uint64_t>(tiles, 2 * resident_grid())), dim3(256), 0, stream, a);
        if (launches) *launches += 1;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace salus
