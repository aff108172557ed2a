// One token from every row of logits: temperature, top-k, top-p, min-p, a given random number.
//
//   order of a row: by logit, equal ones by index;   w = exp((logit - largest) / temperature)
//   kept: the first top_k; of these the fewest from the front whose w reach top_p of their sum; of these those with w >= min_p
//   token: the smallest index up to which the sum of the kept w exceeds u times the sum of all kept
//
// Every limit keeps a beginning of the order, so nothing is sorted: the place of a token in the order is a 52-bit number (the logit's bits, made
// monotonous, in front of the index), and a limit is the number of the last token that is kept, found eleven bits at a time by histograms of how many tokens
// there are, or how much weight.  Weights are 64-bit exponentials, counted as whole multiples of 2^-44: their sums are the same in any order,
// so that atomic additions do not show, and off by less than 2^-25 of the largest weight for 2^19 tokens.
#include "answer.hpp"

namespace salus {

constexpr uint32_t kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64, kBins = 2048;
constexpr double kWeightUnit = 17592186044416.0;      // 2^44

// Units of eight logits of a row.
template <bool BF16>
struct LogitRow {
    const Global<char> *at;
    uint32_t V;
    __device__ uint32_t units() const { return (V + 7) / 8; }
    // What is no logit, and NaN, become minus infinity; minus zero becomes zero.
    __device__ void load(uint32_t unit, float (&x)[8]) const
    {
        if constexpr (BF16) {
            const u32x4 w = *(const Global<u32x4> *)(at + (uint64_t)unit * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = bf16_low(w[i]);
                x[2 * i + 1] = bf16_high(w[i]);
            }
        } else {
            const f32x4 a = *(const Global<f32x4> *)(at + (uint64_t)unit * 32), b = *(const Global<f32x4> *)(at + (uint64_t)unit * 32 + 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = a[i];
                x[4 + i] = b[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = unit * 8 + i < V && x[i] == x[i] ? x[i] + 0.0f : -INFINITY;
    }
};

// A token's place in the order, 52 bits: larger is earlier.
constexpr uint32_t kPlaceBits = 52;
__device__ inline uint64_t place_of(float x, uint32_t index)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 20 | (0xfffffu - index);
}
__device__ inline uint32_t index_of(uint64_t place) { return 0xfffffu - ((uint32_t)place & 0xfffffu); }
__device__ inline float logit_of(uint64_t place)
{
    const uint32_t b = (uint32_t)(place >> 20);
    return __builtin_bit_cast(float, b & 0x80000000u ? b & 0x7fffffffu : ~b);
}

__device__ inline uint64_t wave_max_u64(uint64_t v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, d, 64));
    return v;
}
__device__ inline uint64_t wave_sum_u64(uint64_t v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor((unsigned long long)v, d, 64);
    return v;
}

struct RowLimits {
    float top;                   // largest logit
    double per_temperature;
    uint64_t first;              // place of the first token
    uint64_t cut;                // place of the last token that is kept by top_k and top_p
    double min_p;
    __device__ double weight(float x) const { return x == top ? 1.0 : top == INFINITY ? 0.0 : exp(((double)x - (double)top) * per_temperature); }
    __device__ uint64_t units(double w) const { return (uint64_t)(w * kWeightUnit + 0.5); }
    __device__ uint64_t kept(float x, uint32_t index) const
    {
        if (place_of(x, index) < cut || x == -INFINITY) return 0;
        const double w = weight(x);
        return w >= min_p ? units(w) : 0;
    }
};

struct SampleShared {
    unsigned long long mass[kBins];
    uint32_t count[kBins];
    uint64_t part[kSampleWaves];
    uint64_t before, prefix;
    uint32_t single, token;
};

// Sum, or largest, of every thread's number.
template <bool MAX>
__device__ inline uint64_t block_u64(uint64_t v, SampleShared &s)
{
    v = MAX ? wave_max_u64(v) : wave_sum_u64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (uint32_t i = 0; i < kSampleWaves; ++i) all = MAX ? max(all, s.part[i]) : all + s.part[i];
    return all;
}

// The place of the token with which the first ones of the order reach `target`, tokens or weight (WEIGHT), among those down to l.cut.
template <bool BF16, bool WEIGHT>
__device__ inline uint64_t reach(const LogitRow<BF16> &row, const RowLimits &l, uint64_t target, SampleShared &s)
{
    uint64_t prefix = 0;                     // the bits known so far
    uint32_t left = kPlaceBits;
    for (;;) {
        const uint32_t bits = min(left, 11u), rest = left - bits;
        for (uint32_t i = threadIdx.x; i < kBins; i += kSampleThreads) {
            s.mass[i] = 0;
            s.count[i] = 0;
        }
        __syncthreads();
        for (uint32_t unit = threadIdx.x; unit < row.units(); unit += kSampleThreads) {
            float x[8];
            row.load(unit, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t place = place_of(x[i], unit * 8 + i);
                if (place < l.cut || x[i] == -INFINITY || (left < kPlaceBits && place >> left != prefix)) continue;
                const uint32_t bin = kBins - 1 - ((uint32_t)(place >> rest) & ((1u << bits) - 1));
                atomicAdd(&s.count[bin], 1u);
                if (WEIGHT) atomicAdd(&s.mass[bin], (unsigned long long)l.units(l.weight(x[i])));
            }
        }
        __syncthreads();
        // two bins a thread, the earliest tokens in front
        const uint32_t b = 2 * threadIdx.x;
        const uint64_t n0 = WEIGHT ? s.mass[b] : s.count[b], n1 = WEIGHT ? s.mass[b + 1] : s.count[b + 1];
        uint64_t total;
        uint64_t before = wave_excl_scan_u64(n0 + n1, &total);
        if ((threadIdx.x & 63) == 0) s.part[threadIdx.x >> 6] = total;
        __syncthreads();
        for (uint32_t i = 0; i < threadIdx.x >> 6; ++i) before += s.part[i];
        const bool one = before < target && target <= before + n0, two = before + n0 < target && target <= before + n0 + n1;
        if (one || two) {
            const uint32_t bin = b + two;
            s.before = before + (two ? n0 : 0);
            s.prefix = (left < kPlaceBits ? prefix << bits : 0) | ((kBins - 1 - bin) & ((1u << bits) - 1));
            s.single = s.count[bin] == 1;
        }
        __syncthreads();
        prefix = s.prefix;
        target -= s.before;
        left = rest;
        const bool done = s.single || left == 0;
        __syncthreads();
        if (done) return prefix << left;
    }
}

template <bool BF16>
__device__ inline int32_t sample_row(const SampleProblem &p, uint32_t r, SampleShared &s)
{
    const LogitRow<BF16> row{(const Global<char> *)p.logits + (uint64_t)r * p.ld * (BF16 ? 2 : 4), p.V};
    const u32x4 params = *(const Global<u32x4> *)((const Global<uint32_t> *)p.params + 4 * (uint64_t)r);
    const float temperature = as_float(params[0]), top_p = as_float(params[2]), min_p = as_float(params[3]), u = ((const Global<float> *)p.u)[r];
    const int32_t top_k = (int32_t)params[1];
    uint64_t first = 0;
    for (uint32_t unit = threadIdx.x; unit < row.units(); unit += kSampleThreads) {
        float x[8];
        row.load(unit, x);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (x[i] != -INFINITY) first = max(first, place_of(x[i], unit * 8 + i));
    }
    first = block_u64<true>(first, s);
    if (first == 0) return -1;
    if (!(temperature > 0.0f) || top_k == 1) return (int32_t)index_of(first);
    RowLimits l{logit_of(first), 1.0 / (double)temperature, first, 0, min_p > 0.0f ? fmin(1.0, (double)min_p) : 0.0};
    const auto sum_kept = [&](bool limits) {
        uint64_t sum = 0;
        for (uint32_t unit = threadIdx.x; unit < row.units(); unit += kSampleThreads) {
            float x[8];
            row.load(unit, x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sum += limits ? l.kept(x[i], unit * 8 + i) : place_of(x[i], unit * 8 + i) >= l.cut && x[i] != -INFINITY ? l.units(l.weight(x[i])) : 0;
        }
        return block_u64<false>(sum, s);
    };
    if (top_k > 0 && (uint32_t)top_k < p.V) {
        // logits of minus infinity have no place: fewer may be left
        uint64_t count = 0;
        for (uint32_t unit = threadIdx.x; unit < row.units(); unit += kSampleThreads) {
            float x[8];
            row.load(unit, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) count += x[i] != -INFINITY;
        }
        count = block_u64<false>(count, s);
        if ((uint32_t)top_k < count) l.cut = reach<BF16, false>(row, l, (uint32_t)top_k, s);
    }
    if (top_p < 1.0f) {
        const uint64_t total = sum_kept(false);
        const double want = ceil(fmax((double)top_p, 0.0) * (double)total);
        l.cut = max(l.cut, reach<BF16, true>(row, l, min(max((uint64_t)want, (uint64_t)1), total), s));
    }
    // in order of index: a wavefront has a run of units
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, run = (row.units() + kSampleWaves - 1) / kSampleWaves;
    const uint32_t from = wave * run, to = min(from + run, row.units());
    uint64_t sum = 0;
    for (uint32_t unit = from + lane; unit < to; unit += 64) {
        float x[8];
        row.load(unit, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += l.kept(x[i], unit * 8 + i);
    }
    sum = wave_sum_u64(sum);
    __syncthreads();
    if (lane == 0) s.part[wave] = sum;
    __syncthreads();
    uint64_t all = 0, before = 0;
    for (uint32_t i = 0; i < kSampleWaves; ++i) {
        if (i == wave) before = all;
        all += s.part[i];
    }
    // u of NaN and below 0 is 0; the product is below the sum also where it is rounded up
    const uint64_t target = min((uint64_t)(fmin(fmax((double)u, 0.0), 1.0) * (double)all), all - 1);
    if (before <= target && target < before + sum) {
        for (uint32_t step = from; step < to; step += 64) {
            uint64_t w[8], mine = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 0;
            const uint32_t unit = step + lane;
            if (unit < to) {
                float x[8];
                row.load(unit, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) mine += w[i] = l.kept(x[i], unit * 8 + i);
            }
            uint64_t total, at = before + wave_excl_scan_u64(mine, &total);
            if (at <= target && target < at + mine) {
                uint32_t token = unit * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (at <= target && target < at + w[i]) token = unit * 8 + i;
                    at += w[i];
                }
                s.token = token;
            }
            before += total;
            if (before > target) break;
        }
    }
    __syncthreads();
    return (int32_t)s.token;
}

template <typename Args>
__global__ __launch_bounds__(kSampleThreads) void sample_rows(Args a)
{
    __shared__ SampleShared s;
    SampleProblem p;
    const uint32_t r = find_owner(a.first, a.p, a.base + blockIdx.x, p);
    const int32_t token = p.bf16 ? sample_row<true>(p, r, s) : sample_row<false>(p, r, s);
    if (threadIdx.x == 0) ((Global<int32_t> *)p.tokens)[r] = token;
}

uint64_t sample_work_bytes(uint32_t M, uint32_t) { return 16ull * M; }

hipError_t launch_sample(const SampleProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    const auto rows = [](const SampleProblem &q) { return (uint64_t)q.M; };
    if (n <= kAnswerFew) return launch_answer_of<SampleProblem, kAnswerFew>(sample_rows, kSampleThreads, p, n, stream, launches, rows);
    return launch_answer_of<SampleProblem, kAnswerProblems>(sample_rows, kSampleThreads, p, n, stream, launches, rows);
}

}  // namespace salus
