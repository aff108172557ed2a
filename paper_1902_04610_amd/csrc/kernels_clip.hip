// Global gradient norm of every job of a round and what is done with it: gradients scaled in place, or taken off the float weights.
//
//   norm = sqrt(sum of g^2 over all elements of all the job's tensors),  c = min(1, max_norm / norm)  (a NaN stays one)
//   clip:      g <- g c                 clip_sgd:  wm <- wm - lr (c g),  wb <- bf16(wm)
//
// Two passes, as no gradient can be scaled before all of them have been read; bound by memory in both.  The first writes one sum
// per chunk of a tensor, at most 1024 of them per job beside one per tensor; every workgroup of the second adds its job's chunks
// again in the same order, which costs less than a launch in between.  Squares and sums are held in 64 bits: a square of a float may pass
// the largest float, and the order of the additions then does not show in the result.
#include <algorithm>
#include <vector>

#include "block.hpp"

namespace salus {

constexpr uint32_t kClipTensors = 64, kClipJobs = 32;      // of a launch
constexpr uint64_t kClipCount = (1ull << 48) - 1;
struct ClipEntry {
    void *g;
    float *wm;
    void *wb;
    uint64_t count;          // bits 0-47: elements, 48-55: job, 63: bf16
};
struct ClipOwner {
    double *work;
    float *norm;
    uint32_t sums;           // of the job
    uint32_t shift;          // a chunk is 1 << (kClipChunkBits + shift) elements
    float max_norm, lr;
};
struct ClipArgs {
    uint32_t n, tiles, pad[2];
    uint32_t first[kClipTensors];      // first chunk of tensor i in this launch; kNoTile from n on
    uint32_t at[kClipTensors];         // its number among the job's
    ClipEntry p[kClipTensors];
    ClipOwner job[kClipJobs];
};
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments are limited to 4 KB");

__device__ inline double wave_sum_f64(double v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Sum over the 256 threads of a workgroup, in every thread.
__device__ inline double block_sum_f64(double v)
{
    __shared__ double part[4];
    v = wave_sum_f64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

__device__ inline double square(float v) { return (double)v * (double)v; }

template <bool BF16>
__device__ inline double sum_of_squares(const void *g, uint64_t begin, uint64_t end)
{
    constexpr uint32_t kVec = BF16 ? 8 : 4, kLoads = 4;
    double s[4] = {0, 0, 0, 0};
    // Squares of bf16 numbers are exact in float, and eight of them are added there if that can neither overflow nor lose all of them: 64-bit conversions
    // of every element take longer than reading it.
    auto add = [&](u32x4 w) {
        if constexpr (BF16) {
            float v[8], most = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = bf16_low(w[i]);
                v[2 * i + 1] = bf16_high(w[i]);
                most = fmaxf(most, fmaxf(fabsf(v[2 * i]), fabsf(v[2 * i + 1])));
            }
            float q = v[0] * v[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) q = fmaf(v[i], v[i], q);
            if (most > 0x1p-50f && most < 0x1p50f) {      // not so of a NaN beside ordinary numbers: q is one then
                s[0] += (double)q;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += square(v[2 * i]) + square(v[2 * i + 1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += square(as_float(w[i]));
        }
    };
    const uint64_t whole = begin + (end - begin) / kVec * kVec;
    const Global<char> *base = (const Global<char> *)g;
    constexpr uint32_t kSize = BF16 ? 2 : 4;
    uint64_t i = begin + (uint64_t)kVec * threadIdx.x;
    for (; i + (kLoads - 1) * kVec * 256ull < whole; i += kLoads * kVec * 256) {
        u32x4 w[kLoads];
#pragma unroll
        for (uint32_t l = 0; l < kLoads; ++l) w[l] = *(const Global<u32x4> *)(base + (i + l * kVec * 256ull) * kSize);
#pragma unroll
        for (uint32_t l = 0; l < kLoads; ++l) add(w[l]);
    }
    for (; i < whole; i += kVec * 256) add(*(const Global<u32x4> *)(base + i * kSize));
    const uint64_t rest = whole + threadIdx.x;
    if (rest < end) {
        if constexpr (BF16) s[0] += square(bf16_low(((const Global<uint16_t> *)g)[rest]));
        else s[0] += square(((const Global<float> *)g)[rest]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}

struct ClipChunkOf {
    uint64_t begin, end;
    uint32_t job, chunk, tensor;
    bool bf16;
};
__device__ inline ClipChunkOf find_chunk(const ClipArgs &a, uint32_t id)
{
    const int t = __builtin_amdgcn_readfirstlane(wave_find_range(a.first[threadIdx.x & 63], id, true));
    const uint64_t packed = a.p[t].count, count = packed & kClipCount;
    const uint32_t job = (uint32_t)(packed >> 48) & 0xffu, c = id - a.first[t];
    const uint64_t size = 1ull << (kClipChunkBits + a.job[job].shift), begin = c * size;
    return {begin, min(begin + size, count), job, a.at[t] + c, (uint32_t)t, (packed >> 63) != 0};
}

__global__ __launch_bounds__(256) void clip_norm(ClipArgs a)
{
    const ClipChunkOf c = find_chunk(a, blockIdx.x);
    const void *g = a.p[c.tensor].g;
    const double sum = block_sum_f64(c.bf16 ? sum_of_squares<true>(g, c.begin, c.end) : sum_of_squares<false>(g, c.begin, c.end));
    if (threadIdx.x == 0) ((Global<double> *)a.job[c.job].work)[c.chunk] = sum;
}

// A job's norm, in every thread.
__device__ inline double clip_total(const ClipOwner &job)
{
    double s = 0;
    for (uint32_t i = threadIdx.x; i < job.sums; i += 256) s += ((const Global<double> *)job.work)[i];
    return sqrt(block_sum_f64(s));
}

template <bool BF16, bool SGD>
__device__ inline void apply_clip(const ClipEntry &t, uint64_t begin, uint64_t end, float c, float lr)
{
    constexpr uint32_t kVec = BF16 ? 8 : 4;
    auto one = [&](uint64_t i) {
        float v = BF16 ? bf16_low(((const Global<uint16_t> *)t.g)[i]) : ((const Global<float> *)t.g)[i];
        v = __fmul_rn(v, c);
        if constexpr (SGD) {
            const float w = __fsub_rn(((const Global<float> *)t.wm)[i], __fmul_rn(lr, v));
            ((Global<float> *)t.wm)[i] = w;
            ((Global<uint16_t> *)t.wb)[i] = (uint16_t)bf16_bits(w);
        } else if constexpr (BF16) ((Global<uint16_t> *)t.g)[i] = (uint16_t)bf16_bits(v);
        else ((Global<float> *)t.g)[i] = v;
    };
    constexpr uint32_t kLoads = SGD ? 2 : 4;      // vectors on their way per thread
    const uint64_t whole = begin + (end - begin) / kVec * kVec;
    struct Vec { u32x4 g; f32x4 m[SGD ? kVec / 4 : 1]; };
    auto load = [&](Vec &x, uint64_t i) {
        x.g = *(const Global<u32x4> *)((const Global<char> *)t.g + i * (BF16 ? 2 : 4));
        if constexpr (SGD) {
#pragma unroll
            for (uint32_t q = 0; q < kVec / 4; ++q) x.m[q] = *(const Global<f32x4> *)((const Global<float> *)t.wm + i + 4 * q);
        }
    };
    auto store = [&](const Vec &x, uint64_t i) {
        float v[kVec];
#pragma unroll
        for (uint32_t e = 0; e < kVec; ++e) v[e] = __fmul_rn(BF16 ? (e & 1 ? bf16_high(x.g[e / 2]) : bf16_low(x.g[e / 2])) : as_float(x.g[e & 3]), c);
        if constexpr (SGD) {
            uint32_t b[kVec / 2];
#pragma unroll
            for (uint32_t q = 0; q < kVec; q += 4) {
                f32x4 m = x.m[q / 4];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) m[e] = __fsub_rn(m[e], __fmul_rn(lr, v[q + e]));      // one rounding each
                *(Global<f32x4> *)((Global<float> *)t.wm + i + q) = m;
                b[q / 2] = bf16_pack(m[0], m[1]);
                b[q / 2 + 1] = bf16_pack(m[2], m[3]);
            }
            if constexpr (BF16) *(Global<u32x4> *)((Global<uint16_t> *)t.wb + i) = u32x4{b[0], b[1], b[2], b[3]};
            else *(Global<u32x2> *)((Global<uint16_t> *)t.wb + i) = u32x2{b[0], b[1]};
        } else if constexpr (BF16) {
            *(Global<u32x4> *)((Global<uint16_t> *)t.g + i) = u32x4{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7])};
        } else {
            *(Global<f32x4> *)((Global<float> *)t.g + i) = f32x4{v[0], v[1], v[2], v[3]};
        }
    };
    constexpr uint64_t kStride = kVec * 256;
    uint64_t i = begin + (uint64_t)kVec * threadIdx.x;
    for (; i + (kLoads - 1) * kStride < whole; i += kLoads * kStride) {
        Vec x[kLoads];
#pragma unroll
        for (uint32_t l = 0; l < kLoads; ++l) load(x[l], i + l * kStride);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t l = 0; l < kLoads; ++l) store(x[l], i + l * kStride);
    }
    for (; i < whole; i += kStride) {
        Vec x;
        load(x, i);
        store(x, i);
    }
    if (whole + threadIdx.x < end) one(whole + threadIdx.x);
}

template <bool SGD>
__global__ __launch_bounds__(256) void clip_apply(ClipArgs a)
{
    const ClipChunkOf c = find_chunk(a, blockIdx.x);
    const ClipOwner &job = a.job[c.job];
    const double norm = clip_total(job), ratio = (double)job.max_norm / norm;
    if (c.chunk == 0 && threadIdx.x == 0) *(Global<float> *)job.norm = (float)norm;
    const float scale = (float)(ratio > 1.0 ? 1.0 : ratio);
    const ClipEntry &t = a.p[c.tensor];
    // nothing is scaled below the limit: x 1 would write back what is there
    if (!SGD && scale == 1.0f) return;
    if (c.bf16) apply_clip<true, SGD>(t, c.begin, c.end, scale, job.lr);
    else apply_clip<false, SGD>(t, c.begin, c.end, scale, job.lr);
}

hipError_t launch_clip(const ClipJob *jobs, uint32_t n, bool sgd, hipStream_t stream, uint64_t *launches)
{
    std::vector<ClipArgs> parts;
    parts.reserve(8);
    uint32_t used = kClipJobs;      // jobs in the last part
    for (uint32_t j = 0; j < n; ++j) {
        const ClipJob &job = jobs[j];
        uint64_t sums = 0;
        const uint32_t shift = clip_shift(job.n_tensors, [&](uint32_t i) { return job.tensors[i].count; }, &sums);
        const ClipOwner owner = {job.work, job.norm, (uint32_t)sums, shift, job.max_norm, job.lr};
        uint64_t at = 0;
        bool entered = false;
        for (uint32_t i = 0; i < job.n_tensors; ++i) {
            const ClipTensor &t = job.tensors[i];
            const uint64_t count = clip_chunks(t.count, shift);
            if (parts.empty() || parts.back().n == kClipTensors || (!entered && used == kClipJobs) || parts.back().tiles + count > 0x7fffffffull) {
                parts.push_back(ClipArgs{});
                for (uint32_t &f : parts.back().first) f = kNoTile;
                used = 0;
                entered = false;
            }
            ClipArgs &a = parts.back();
            if (!entered) {
                a.job[used++] = owner;
                entered = true;
            }
            a.p[a.n] = {t.g, t.wm, t.wb, t.count | (uint64_t)(used - 1) << 48 | (uint64_t)(t.bf16 != 0) << 63};
            a.first[a.n] = a.tiles;
            a.at[a.n] = (uint32_t)at;
            a.n += 1;
            a.tiles += (uint32_t)count;
            at += count;
        }
    }
    for (int pass = 0; pass < 2; ++pass)
        for (const ClipArgs &a : parts) {
            if (pass == 0) hipLaunchKernelGGL(clip_norm, dim3(a.tiles), dim3(256), 0, stream, a);
            else if (sgd) hipLaunchKernelGGL(clip_apply<true>, dim3(a.tiles), dim3(256), 0, stream, a);
            else hipLaunchKernelGGL(clip_apply<false>, dim3(a.tiles), dim3(256), 0, stream, a);
            if (launches) *launches += 1;
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace salus
