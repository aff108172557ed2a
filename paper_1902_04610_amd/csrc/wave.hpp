// Wavefront-level (64-lane) primitives shared by the kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace salus {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A T in device memory, for addresses the compiler cannot trace to a kernel argument (it would use flat accesses,
// which count as LDS accesses too and are waited for in order).
template <typename T>
using Global = T __attribute__((address_space(1)));

// Exclusive prefix sum across the 64 lanes of a wavefront (Hillis-Steele over
// cross-lane shuffles).  *total receives the sum over all lanes.
__device__ inline uint64_t wave_excl_scan_u64(uint64_t v, uint64_t *total)
{
    const int lane = threadIdx.x & 63;
    uint64_t incl = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        uint64_t up = __shfl_up((unsigned long long)incl, d, 64);
        if (lane >= d) incl += up;
    }
    if (total) *total = __shfl((unsigned long long)incl, 63, 64);
    return incl - v;
}

// Index of the lane whose half-open range [excl, excl + count) contains x, given
// each lane's exclusive prefix and the number of valid lanes.  Lanes with an
// empty range never win.  x must be below the total.
__device__ inline int wave_find_range(uint64_t excl, uint64_t x, bool valid)
{
    unsigned long long m = __ballot(valid && excl <= x);
    return 63 - __clzll((long long)m);
}

// Sums and maxima across the lanes by data-parallel moves (row shifts by 1, 2, 4, 8, then the last lane of a row, or of two, to the rows behind it): some ten cycles a step, where
// a shuffle takes a hundred.  T: any type of 4 or 8 bytes whose zero is all bits zero; lanes without a source get zero.
template <int CONTROL, int ROWS, typename T>
__device__ inline T lanes_from(T v)
{
    static_assert(sizeof(T) == 4 || sizeof(T) == 8, "words");
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, ROWS, 0xf, false));
    } else {
        const uint64_t w = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CONTROL, ROWS, 0xf, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CONTROL, ROWS, 0xf, false);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    }
}
template <typename T, typename Op>
__device__ inline T wave_scan(T v, Op op)      // of the lanes up to this one
{
    v = op(v, lanes_from<0x111, 0xf>(v));
    v = op(v, lanes_from<0x112, 0xf>(v));
    v = op(v, lanes_from<0x114, 0xf>(v));
    v = op(v, lanes_from<0x118, 0xf>(v));
    v = op(v, lanes_from<0x142, 0xa>(v));
    return op(v, lanes_from<0x143, 0xc>(v));
}
// Lane `lane`'s (the same one in all lanes) v.
template <typename T>
__device__ inline T lane_value(T v, uint32_t lane)
{
    static_assert(sizeof(T) == 4 || sizeof(T) == 8, "words");
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const uint64_t w = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)w, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(w >> 32), lane);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    }
}
template <typename T>
__device__ inline T wave_sum_scan(T v) { return wave_scan(v, [](T a, T b) { return a + b; }); }
template <typename T>
__device__ inline T wave_total(T v) { return lane_value(wave_sum_scan(v), 63); }
template <typename T>
__device__ inline T wave_largest(T v) { return lane_value(wave_scan(v, [](T a, T b) { return a > b ? a : b; }), 63); }      // unsigned

}  // namespace salus
