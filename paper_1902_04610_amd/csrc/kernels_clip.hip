// Global gradient norm of every job of a round and what is done with it: gradients scaled in place, or taken off the float weights.
//
//   norm = sqrt(sum of g^2 over all elements of all the job's tensors),  c = min(1, max_norm / norm)  (a NaN stays one)
//   clip:      g <- g c                 clip_sgd:  wm <- wm - lr (c g),  wb <- bf16(wm)
//
// Two passes, as no gradient can be scaled before all of them have been read; bound by memory in both.  Tensors are read in chunks of 4096 elements, which a job's
// workgroups take in turn, so that all of them together sweep through memory: what is under way at a time is a few windows, not a thousand.  The first
// pass writes one sum per workgroup; every workgroup of the second adds its job's sums again, in the same order, which costs
// less than a launch in between, and goes from the last chunk to the first, whose gradients the memory-side cache still holds.  Squares and sums are held in 64 bits: a
// square of a float may pass the largest float, and the order of the additions then does not show in the result.
#include <algorithm>
#include <iterator>
#include <vector>

#include "block.hpp"

namespace salus {

constexpr uint32_t kClipThreads = 256, kClipJobs = 32;      // of a workgroup, of a launch
constexpr uint64_t kClipCount = (1ull << 48) - 1, kClipChunk = 1ull << kClipChunkBits;
struct ClipEntry {
    void *g;
    float *wm;
    void *wb;
    uint64_t count;          // bits 0-47: elements; 63: bf16
};
struct ClipOwner {
    double *work;
    float *norm;             // null but in the launch of the job's first tensor
    uint32_t sums;           // of the job, in all launches
    uint32_t at;             // of them, where those of this launch begin
    uint32_t begin, end;     // its chunks in this launch
    uint32_t block, blocks;  // its workgroups
    float max_norm, lr;
};
template <uint32_t TENSORS, uint32_t JOBS>
struct ClipArgsOf {
    uint32_t n, tiles, jobs, blocks;
    uint32_t first[TENSORS];      // first chunk of tensor i; kNoTile from n on
    ClipEntry p[TENSORS];
    ClipOwner job[JOBS];
};
typedef ClipArgsOf<kClipTensors, kClipJobs> ClipArgs;
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments are limited to 4 KB");
// The same for launches of few tensors, whose time is the host's.
typedef ClipArgsOf<16, 4> ClipFewArgs;

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
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

__device__ inline double square(float v) { return (double)v * (double)v; }

// The squares of 16 bytes, in 64 bits whatever the type: eight squares of bf16 numbers added in float would lose all that are below 2^-24 of the first.
template <bool BF16>
__device__ inline double squares(u32x4 w)
{
    if constexpr (BF16) {
        double low = 0, high = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            low += square(bf16_low(w[i]));
            high += square(bf16_high(w[i]));
        }
        return low + high;
    } else {
        return (square(as_float(w[0])) + square(as_float(w[1]))) + (square(as_float(w[2])) + square(as_float(w[3])));
    }
}

// Which job a workgroup works for, and the chunks of the launch: lane i holds the first of tensor i.
struct ClipChunk { const ClipEntry *t; uint64_t begin, end; bool bf16; };
template <typename Args>
struct ClipWalk {
    static constexpr uint32_t kTensors = sizeof(Args::first) / 4, kJobs = sizeof(Args::job) / sizeof(ClipOwner);
    const Args &a;
    const uint32_t first;
    int job;
    uint32_t mine;       // this workgroup's number among the job's
    __device__ explicit ClipWalk(const Args &args) : a(args), first(args.first[min(threadIdx.x & 63, kTensors - 1)])
    {
        const uint32_t lane = threadIdx.x & 63;
        job = __builtin_amdgcn_readfirstlane(wave_find_range(a.job[min(lane, kJobs - 1)].block, blockIdx.x, lane < a.jobs));
        mine = blockIdx.x - a.job[job].block;
    }
    __device__ ClipChunk chunk(uint32_t c) const
    {
        const int t = __builtin_amdgcn_readfirstlane(wave_find_range(first, c, (threadIdx.x & 63) < a.n));
        const uint64_t count = a.p[t].count & kClipCount, begin = (uint64_t)(c - (uint32_t)__builtin_amdgcn_readlane(first, t)) << kClipChunkBits;
        return {&a.p[t], begin, min(begin + kClipChunk, count), (a.p[t].count >> 63) != 0};
    }
};

// The squares of C whole chunks of one type, every load asked for at once (a thread has 16 elements of each).
template <bool BF16, int C>
__device__ inline double whole_chunks(const ClipChunk (&c)[C])
{
    constexpr uint32_t kVec = BF16 ? 8 : 4, kSize = BF16 ? 2 : 4, V = kClipChunk / kClipThreads / kVec;
    u32x4 w[C][V];
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (uint32_t v = 0; v < V; ++v)
            w[i][v] = *(const Global<u32x4> *)((const Global<char> *)c[i].t->g + (c[i].begin + kVec * (threadIdx.x + v * kClipThreads)) * kSize);
    double s = 0;
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (uint32_t v = 0; v < V; ++v) s += squares<BF16>(w[i][v]);
    return s;
}

template <bool BF16>
__device__ inline double chunk_squares(const ClipChunk &c)
{
    constexpr uint32_t kVec = BF16 ? 8 : 4, kSize = BF16 ? 2 : 4;
    if (c.end - c.begin == kClipChunk) return whole_chunks<BF16, 1>({c});
    const Global<char> *g = (const Global<char> *)c.t->g;
    double s = 0;
    const uint64_t whole = c.begin + (c.end - c.begin) / kVec * kVec;
    for (uint64_t j = c.begin + kVec * threadIdx.x; j < whole; j += kVec * kClipThreads) s += squares<BF16>(*(const Global<u32x4> *)(g + j * kSize));
    if (whole + threadIdx.x < c.end) {
        if constexpr (BF16) s += square(bf16_low(((const Global<uint16_t> *)g)[whole + threadIdx.x]));
        else s += square(((const Global<float> *)g)[whole + threadIdx.x]);
    }
    return s;
}

// Two chunks at a time: one alone leaves too few loads under way where one job has the launch (370 MB: 69 us with one, 62 with two workgroups where there is one now).
template <typename Args>
__global__ __launch_bounds__(kClipThreads) void clip_norm(Args a)
{
    const ClipWalk<Args> walk(a);
    const ClipOwner &job = a.job[walk.job];
    double s = 0;
    uint32_t c = job.begin + walk.mine;
    for (; c + (uint64_t)job.blocks < job.end; c += 2 * job.blocks) {
        const ClipChunk k[2] = {walk.chunk(c), walk.chunk(c + job.blocks)};
        const bool both = k[0].end - k[0].begin == kClipChunk && k[1].end - k[1].begin == kClipChunk && k[0].bf16 == k[1].bf16;
        if (both) s += k[0].bf16 ? whole_chunks<true, 2>(k) : whole_chunks<false, 2>(k);
        else
            for (const ClipChunk &one : k) s += one.bf16 ? chunk_squares<true>(one) : chunk_squares<false>(one);
    }
    if (c < job.end) {
        const ClipChunk k = walk.chunk(c);
        s += k.bf16 ? chunk_squares<true>(k) : chunk_squares<false>(k);
    }
    s = block_sum_f64(s);
    if (threadIdx.x == 0) ((Global<double> *)job.work)[job.at + walk.mine] = s;
}

// A job's norm, in every thread.
__device__ inline double clip_total(const ClipOwner &job)
{
    double s = 0;
    for (uint32_t i = threadIdx.x; i < job.sums; i += kClipThreads) s += ((const Global<double> *)job.work)[i];
    return sqrt(block_sum_f64(s));
}

// Vectors are as wide as the widest of what lies beside them allows to be read and written in whole lines: four elements with float weights.
// PAST: what the call moves does not fit the memory-side cache, and goes past the caches (non-temporal): 8 jobs x 25 M elements, bf16 gradients,
// 455 / 482 us and the norms of the next call, behind stores that are still under way, 71 / 124.
template <bool BF16, bool SGD, bool PAST>
__device__ inline void apply_clip(const ClipChunk &k, float c, float lr)
{
    constexpr uint32_t kVec = BF16 && !SGD ? 8 : 4, V = kClipChunk / kClipThreads / kVec, kWords = BF16 ? kVec / 2 : kVec;
    typedef uint32_t words __attribute__((ext_vector_type(kWords)));
    const ClipEntry &t = *k.t;
    struct Vec { words g; f32x4 m; };
    auto load = [&](Vec &x, uint64_t i) {
        const Global<words> *g = (const Global<words> *)((const Global<char> *)t.g + i * (BF16 ? 2 : 4));
        x.g = PAST ? __builtin_nontemporal_load(g) : *g;
        if constexpr (SGD) {
            const Global<f32x4> *m = (const Global<f32x4> *)((const Global<float> *)t.wm + i);
            x.m = PAST ? __builtin_nontemporal_load(m) : *m;
        }
    };
    auto put = [](auto v, auto *to) {
        if constexpr (PAST) __builtin_nontemporal_store(v, to);
        else *to = v;
    };
    auto store = [&](const Vec &x, uint64_t i) {
        float v[kVec];
#pragma unroll
        for (uint32_t e = 0; e < kVec; ++e) v[e] = __fmul_rn(BF16 ? (e & 1 ? bf16_high(x.g[e / 2]) : bf16_low(x.g[e / 2])) : as_float(x.g[e & (kWords - 1)]), c);
        if constexpr (SGD) {
            f32x4 m;
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) m[e] = __fsub_rn(x.m[e], __fmul_rn(lr, v[e]));      // one rounding each
            put(m, (Global<f32x4> *)((Global<float> *)t.wm + i));
            put(u32x2{bf16_pack(m[0], m[1]), bf16_pack(m[2], m[3])}, (Global<u32x2> *)((Global<uint16_t> *)t.wb + i));
        } else if constexpr (BF16) {
            put(u32x4{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7])}, (Global<u32x4> *)((Global<uint16_t> *)t.g + i));
        } else {
            put(f32x4{v[0], v[1], v[2], v[3]}, (Global<f32x4> *)((Global<float> *)t.g + i));
        }
    };
    const uint64_t i = k.begin + kVec * threadIdx.x;
    if (k.end - k.begin == kClipChunk) {
        Vec x[V];
#pragma unroll
        for (uint32_t v = 0; v < V; ++v) load(x[v], i + v * kVec * kClipThreads);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t v = 0; v < V; ++v) store(x[v], i + v * kVec * kClipThreads);
        return;
    }
    const uint64_t whole = k.begin + (k.end - k.begin) / kVec * kVec;
    for (uint64_t j = i; j < whole; j += kVec * kClipThreads) {
        Vec x;
        load(x, j);
        store(x, j);
    }
    const uint64_t j = whole + threadIdx.x;
    if (j >= k.end) return;
    float v = BF16 ? bf16_low(((const Global<uint16_t> *)t.g)[j]) : ((const Global<float> *)t.g)[j];
    v = __fmul_rn(v, c);
    if constexpr (SGD) {
        const float w = __fsub_rn(((const Global<float> *)t.wm)[j], __fmul_rn(lr, v));
        ((Global<float> *)t.wm)[j] = w;
        ((Global<uint16_t> *)t.wb)[j] = (uint16_t)bf16_bits(w);
    } else if constexpr (BF16) ((Global<uint16_t> *)t.g)[j] = (uint16_t)bf16_bits(v);
    else ((Global<float> *)t.g)[j] = v;
}

template <bool SGD, bool PAST, typename Args>
__global__ __launch_bounds__(kClipThreads) void clip_apply(Args a)
{
    const ClipWalk<Args> walk(a);
    const ClipOwner &job = a.job[walk.job];
    const double norm = clip_total(job), ratio = norm <= (double)job.max_norm ? 1.0 : (double)job.max_norm / norm;      // no limit: also an infinite norm is within it
    if (job.norm && walk.mine == 0 && threadIdx.x == 0) *(Global<float> *)job.norm = (float)norm;
    const float scale = (float)(ratio > 1.0 ? 1.0 : ratio);
    // nothing is scaled below the limit: x 1 would write back what is there
    if (!SGD && scale == 1.0f) return;
    for (uint32_t c = job.begin + walk.mine; c < job.end; c += job.blocks) {
        const ClipChunk k = walk.chunk(job.begin + job.end - 1 - c);
        if (k.bf16) apply_clip<true, SGD, PAST>(k, scale, job.lr);
        else apply_clip<false, SGD, PAST>(k, scale, job.lr);
    }
}

template <typename Args>
static void launch_pass(const Args &a, bool apply, bool sgd, bool past, hipStream_t stream)
{
    auto go = [&](void (*kernel)(Args)) { hipLaunchKernelGGL(kernel, dim3(a.blocks), dim3(kClipThreads), 0, stream, a); };
    if (!apply) go(clip_norm<Args>);
    else if (sgd) go(past ? clip_apply<true, true, Args> : clip_apply<true, false, Args>);
    else go(past ? clip_apply<false, true, Args> : clip_apply<false, false, Args>);
}

hipError_t launch_clip(const ClipJob *jobs, uint32_t n, bool sgd, hipStream_t stream, uint64_t *launches)
{
    // A job's tensors go in groups of kClipTensors, whatever the other jobs have (so its sums are the same in any company); a group joins the first launch with room.
    std::vector<ClipArgs> parts;
    uint64_t bytes = 0;
    for (uint32_t j = 0; j < n; ++j) {
        const ClipJob &job = jobs[j];
        const uint32_t sums = (uint32_t)clip_sums(job.n_tensors, [&](uint32_t i) { return job.tensors[i].count; });
        for (uint32_t i = 0, at = 0; i < job.n_tensors; i += kClipTensors) {
            const uint32_t count = std::min(kClipTensors, job.n_tensors - i);
            uint64_t chunks = 0;
            for (uint32_t k = 0; k < count; ++k) chunks += clip_chunks(job.tensors[i + k].count);
            if (chunks > 0x7fffffffull) return hipErrorInvalidValue;
            auto part = std::find_if(parts.begin(), parts.end(), [&](const ClipArgs &a) {
                return a.n + count <= kClipTensors && a.jobs < kClipJobs && a.tiles + chunks <= 0x7fffffffull;
            });
            if (part == parts.end()) {
                parts.push_back(ClipArgs{});
                part = parts.end() - 1;
                for (uint32_t &f : part->first) f = kNoTile;
            }
            ClipArgs &a = *part;
            const uint32_t blocks = (uint32_t)std::min<uint64_t>(chunks, kClipSums);
            a.job[a.jobs++] = {job.work, i == 0 ? job.norm : nullptr, sums, at, a.tiles, a.tiles + (uint32_t)chunks, a.blocks, blocks, job.max_norm, job.lr};
            a.blocks += blocks;
            at += blocks;
            for (uint32_t k = 0; k < count; ++k) {
                const ClipTensor &t = job.tensors[i + k];
                bytes += t.count * ((t.bf16 ? 2 : 4) + (sgd ? 6 : 0));
                a.p[a.n] = {t.g, t.wm, t.wb, t.count | (uint64_t)(t.bf16 != 0) << 63};
                a.first[a.n++] = a.tiles;
                a.tiles += (uint32_t)clip_chunks(t.count);
            }
        }
    }
    const bool past = bytes > kCachedBytes;
    ClipFewArgs few{};
    const bool small = parts.size() == 1 && parts[0].n <= sizeof(few.first) / 4 && parts[0].jobs <= sizeof(few.job) / sizeof(ClipOwner);
    if (small) {
        const ClipArgs &a = parts[0];
        few.n = a.n;
        few.tiles = a.tiles;
        few.jobs = a.jobs;
        few.blocks = a.blocks;
        std::copy_n(a.first, std::size(few.first), few.first);
        std::copy_n(a.p, std::size(few.p), few.p);
        std::copy_n(a.job, std::size(few.job), few.job);
    }
    for (int pass = 0; pass < 2; ++pass)
        for (size_t i = 0; i < parts.size(); ++i) {
            if (small) launch_pass(few, pass != 0, sgd, past, stream);
            else launch_pass(parts[pass ? parts.size() - 1 - i : i], pass != 0, sgd, past, stream);
            if (launches) *launches += 1;
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace salus
