// One token from every row of logits: temperature, top-k, top-p, min-p, a given random number.
//
//   order of a row: by logit, equal ones by index;   w = exp((logit - largest) / temperature)
//   kept: the first top_k; of these the fewest from the front whose w reach top_p of their sum; of these those with w >= min_p
//   token: the smallest index up to which the sum of the kept w exceeds u times the sum of all kept
//
// Every limit keeps a beginning of the order, so nothing is sorted: the place of a token in the order is a 52-bit number (the logit's bits, made
// monotonous, in front of the index), and a limit is the number of the last token that is kept.
//
// Two kernels.  Reading the logits once would take 9 us for 256 rows of 128256 bf16; this takes 84 with rows of all kinds of limits (16 for one row of 32000 floats):
//   slice_rows    a workgroup takes 8192 logits of a row and leaves their first token, their sum of weights if the row wants it, and the places of
//                 those that a limit may keep, in order of index: all down to a threshold that at least so many of its threads' largest logits reach as
//                 the limit may want of one slice; for top_p also the weight in bins of 1 / 16 of a power of two.  Bound by its vector instructions: 18 us
//                 for greedy rows, 27 with lists, 40 with 64-bit weights, 56 with bins.
//   choose_rows   a workgroup per row puts that together.  Without limits it reads one slice again (10 us); where the kept tokens all lie above every
//                 slice's threshold, which the lists tell, none (8 - 20).  Else it finds the bin in which top_p ends, reads the row once for that bin's tokens, and one
//                 slice again for the token (43 for one such row: one compute unit's latencies and instructions, a chain of some ten barriers); with min_p too it
//                 reads the row again for the kept weight of sixteen runs.
// What even that does not hold (lists that run over: thousands of equal logits, top_k beyond them, or most of its tokens in one slice) is found by reading the row several times
// (choose_anywhere), eleven bits of the last place at a time by histograms of how many tokens there are, or how much weight: 126 - 220 us for one row of 128256 bf16 with top_k
// 50 - 1000 in one slice (20 - 25 spread evenly), 370 - 383 for 256 of them (46 - 52), with top_p too 325 - 387 and 672 - 688.
//
// Weights are 64-bit exponentials of differences to the row's largest logit, to 1e-11; where they are summed by atomic additions they count as whole multiples of 2^-44, so
// that no order shows.
#include <cfloat>

#include "answer.hpp"

namespace salus {

constexpr uint32_t kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64, kBins = 2048;
constexpr double kWeightUnit = 17592186044416.0;      // 2^44
constexpr uint32_t kSliceThreads = 512, kSliceWaves = kSliceThreads / 64, kSlice = 8192, kListed = 64, kMostListed = 4096, kMassBins = 512;

// What slice_rows leaves of a slice.
struct Slice {
    uint64_t first;          // place of its first token, 0 if it has none
    double mass;             // sum of its weights relative to its first token's
    uint32_t count[kSliceWaves];      // tokens of its wavefronts' lists; more than kListed: the list has not all
    uint32_t down_to;        // the lists have all whose logit's bits (the upper 32 of a place) reach this
    int32_t bin;             // of its first token, if its weights are in bins
    uint32_t binned;
    uint32_t pad;
};
typedef uint32_t SliceWords __attribute__((ext_vector_type(4)));
constexpr uint32_t kSliceWords = sizeof(Slice) / sizeof(SliceWords);
static_assert(kSliceWaves == 8 && kSliceWords == 4, "stored as words");

// Work of a row: its slices, their lists of kListed places for each wavefront, their bins.
__host__ __device__ inline uint32_t slices_of(uint32_t V) { return (V + kSlice - 1) / kSlice; }
struct RowWork {
    Global<char> *at;
    uint32_t slices, units;      // slices, units of each (fewer of the last)
    __host__ __device__ static uint64_t size(uint32_t V) { return (uint64_t)slices_of(V) * (sizeof(Slice) + 8 * kSliceWaves * kListed + 8 * kMassBins); }
    __device__ RowWork(const SampleProblem &p, uint32_t r) : at((Global<char> *)p.work + r * size(p.V)), slices(slices_of(p.V)), units(((p.V + 7) / 8 + slices - 1) / slices) {}
    __device__ Global<SliceWords> *slice(uint32_t i) const { return (Global<SliceWords> *)at + kSliceWords * i; }
    __device__ Global<uint64_t> *list(uint32_t i, uint32_t wave) const { return (Global<uint64_t> *)slice(slices) + (i * kSliceWaves + wave) * kListed; }
    __device__ Global<uint64_t> *bins(uint32_t i) const { return list(slices, 0) + i * kMassBins; }
    __device__ void store(uint32_t i, const Slice &s) const
    {
        Global<SliceWords> *to = slice(i);
        const uint64_t mass = __builtin_bit_cast(uint64_t, s.mass);
        to[0] = SliceWords{(uint32_t)s.first, (uint32_t)(s.first >> 32), (uint32_t)mass, (uint32_t)(mass >> 32)};
        to[1] = SliceWords{s.count[0], s.count[1], s.count[2], s.count[3]};
        to[2] = SliceWords{s.count[4], s.count[5], s.count[6], s.count[7]};
        to[3] = SliceWords{s.down_to, (uint32_t)s.bin, s.binned, 0};
    }
    __device__ Slice load(uint32_t i) const
    {
        const Global<SliceWords> *from = slice(i);
        const SliceWords a = from[0], b = from[1], c = from[2], d = from[3];
        return {(uint64_t)a[1] << 32 | a[0], __builtin_bit_cast(double, (uint64_t)a[3] << 32 | a[2]), {b[0], b[1], b[2], b[3], c[0], c[1], c[2], c[3]}, d[0], (int32_t)d[1], d[2], 0};
    }
};

// A row's logits.  What is no number becomes minus infinity (of a number and NaN the larger is the number), minus zero becomes zero.
struct LogitRow {
    const Global<char> *at;
    uint32_t V, bf16;
    __device__ LogitRow(const SampleProblem &p, uint32_t r) : at((const Global<char> *)p.logits + (uint64_t)r * p.ld * (p.bf16 ? 2 : 4)), V(p.V), bf16(p.bf16) {}
    __device__ uint32_t units() const { return (V + 7) / 8; }
    __device__ static float clean(float x) { return fmaxf(x, -INFINITY) + 0.0f; }
    __device__ float operator[](uint32_t i) const
    {
        return clean(bf16 ? bf16_low(((const Global<uint16_t> *)at)[i]) : ((const Global<float> *)at)[i]);
    }
    // Eight of them.
    struct Raw { u32x4 w[2]; };
    __device__ Raw raw(uint32_t unit) const
    {
        Raw r;
        r.w[0] = *(const Global<u32x4> *)(at + (uint64_t)unit * (bf16 ? 16 : 32));
        if (!bf16) r.w[1] = *(const Global<u32x4> *)(at + (uint64_t)unit * 32 + 16);
        return r;
    }
    __device__ void values(const Raw &r, float (&x)[8]) const      // as they stand there
    {
        if (bf16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i % 2 ? bf16_high(r.w[0][i / 2]) : bf16_low(r.w[0][i / 2]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = as_float(r.w[i / 4][i % 4]);
        }
    }
    __device__ void convert(const Raw &r, uint32_t unit, float (&x)[8]) const
    {
        values(r, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = clean(x[i]);
        if (unit * 8 + 8 > V) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = unit * 8 + i < V ? x[i] : -INFINITY;
        }
    }
};

// A float's bits, made monotonous.
__device__ inline uint32_t key_of(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float float_of(uint32_t key) { return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// A token's place in the order, 52 bits: larger is earlier.
constexpr uint32_t kPlaceBits = 52;
__device__ inline uint64_t place_of(float x, uint32_t index) { return (uint64_t)key_of(x) << 20 | (0xfffffu - index); }
__device__ inline uint32_t index_of(uint64_t place) { return 0xfffffu - ((uint32_t)place & 0xfffffu); }
__device__ inline float logit_of(uint64_t place) { return float_of((uint32_t)(place >> 20)); }

// 2^(d per), the product from -64 to 0, to 1e-11 of itself: the series of 2^f = e^(f ln 2) up to f^9 on [-1/2, 1/2], whose next term is below (ln 2 / 2)^10 / 10! = 7e-12;
// 3 2^51 rounds to whole numbers, which then stand in the lowest bits.
__device__ inline double power_of_two(double d, double per)
{
    constexpr double kWhole = 6755399441055744.0, kLn2 = 0.6931471805599453, k2 = kLn2 * kLn2, k4 = k2 * k2;
    const double whole = fma(d, per, kWhole), f = fma(d, per, kWhole - whole);
    double v = fma(k4 * k4 * kLn2 / 362880, f, k4 * k4 / 40320);
    v = fma(v, f, k4 * k2 * kLn2 / 5040);
    v = fma(v, f, k4 * k2 / 720);
    v = fma(v, f, k4 * kLn2 / 120);
    v = fma(v, f, k4 / 24);
    v = fma(v, f, k2 * kLn2 / 6);
    v = fma(v, f, k2 / 2);
    v = fma(v, f, kLn2);
    v = fma(v, f, 1.0);
    return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, v) + (__builtin_bit_cast(uint64_t, whole) << 52));
}

// Weights relative to a row's, or a slice's, largest logit.
struct Weights {
    float top;
    double per;              // log2(e) / temperature
    __device__ Weights(float t, float temperature) : top(t), per(1.4426950408889634 / (double)temperature) {}
    __device__ double of(float x) const
    {
        const double d = (double)x - (double)top;
        return x == top ? 1.0 : top == INFINITY || !(d * per > -64.0) ? 0.0 : power_of_two(d, per);
    }
};

struct RowLimits : Weights {
    uint64_t first;              // place of the first token
    uint64_t cut;                // place of the last token that is kept by top_k and top_p
    double min_p;
    __device__ RowLimits(uint64_t first_place, float temperature, float min) : Weights(logit_of(first_place), temperature), first(first_place), cut(0), min_p((double)min) {}
    __device__ uint64_t units(double w) const { return (uint64_t)(w * kWeightUnit + 0.5); }
    __device__ uint64_t kept(float x, uint32_t index) const
    {
        if (place_of(x, index) < cut || x == -INFINITY) return 0;
        const double w = of(x);
        return w >= min_p ? units(w) : 0;
    }
};

// A row's parameters.
struct RowParams {
    float temperature, top_p, min_p, u;
    int32_t top_k;           // 0: all
    __device__ RowParams(const SampleProblem &p, uint32_t r)
    {
        const u32x4 w = *(const Global<u32x4> *)((const Global<uint32_t> *)p.params + 4 * (uint64_t)r);
        temperature = as_float(w[0]) > FLT_MAX ? FLT_MAX : as_float(w[0]);
        top_k = max((int32_t)w[1], 0);
        if ((uint32_t)top_k >= p.V) top_k = 0;
        top_p = as_float(w[2]);
        min_p = as_float(w[3]) > 0.0f ? fminf(as_float(w[3]), 1.0f) : 0.0f;
        u = ((const Global<float> *)p.u)[r];
    }
    __device__ bool greedy() const { return !(temperature > 0.0f) || top_k == 1; }
    __device__ bool limited() const { return top_k || top_p < 1.0f || min_p > 0.0f; }
    __device__ bool wants_mass() const { return !greedy() && (top_p < 1.0f ? top_k == 0 : !limited()); }
    // Weight with which top_p is reached, of a total.
    __device__ uint64_t share(double total) const { return max((uint64_t)ceil(fmax((double)top_p, 0.0) * total), (uint64_t)1); }
    // The kept weight in front of the token: u of NaN and below 0 is 0.
    __device__ double before(double total) const { return fmin(fmax((double)u, 0.0), 1.0) * total; }
};

// Bins of weight: numbered by the logit alone, so that those of different slices can be added.  Larger is earlier.
struct BinScale {
    float scale;             // 16 log2(e) / temperature
    __device__ explicit BinScale(float temperature) : scale(16.0f * 1.4426950f / temperature) {}
    __device__ bool usable() const { return scale > 1e-30f && scale < 1e30f; }
    __device__ float raw(float x) const { return fminf(fmaxf(x * scale, -1e6f), 1e6f); }
    __device__ int32_t of(float x) const { return (int32_t)floorf(raw(x)); }      // (all whole numbers of this size are floats)
};

constexpr uint32_t kSliceLoads = kSlice / 8 / kSliceThreads;      // units of a thread
// As Weights::of, but what is below 2^-64 counts as that: 2^(n / 32) 2^f of a table and the series up to f^4 on [-1/64, 1/64], whose next term is below
// (ln 2 / 64)^5 / 5! = 2e-12; 3 2^46 rounds to multiples of 1/32.
constexpr uint32_t kPowers = 32;
struct SliceWeights {
    double top, per, least;
    const double *powers;
    __device__ SliceWeights(float t, float temperature, const double *table) : top(t), per(1.4426950408889634 / (double)temperature), least(-64.0 / per), powers(table) {}
    __device__ static double power(uint32_t i) { return 2.0 * power_of_two((double)i - kPowers, 1.0 / kPowers); }
    __device__ double of(float x) const
    {
        constexpr double kWhole = 211106232532992.0, kLn2 = 0.6931471805599453, k2 = kLn2 * kLn2;
        const double d = fmax((double)x - top, least), whole = fma(d, per, kWhole), f = fma(d, per, kWhole - whole);
        const int32_t n = (int32_t)(uint32_t)__builtin_bit_cast(uint64_t, whole);
        double v = fma(k2 * k2 / 24, f, k2 * kLn2 / 6);
        v = fma(v, f, k2 / 2);
        v = fma(v, f, kLn2);
        v = fma(v, f, 1.0) * powers[n & (int32_t)(kPowers - 1)];
        return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, v) + ((uint64_t)(uint32_t)(n >> 5) << 52));
    }
};

struct SliceShared {
    f32x4 x[2 * kSliceLoads * kSliceThreads];      // a thread's j-th unit: four logits at 2 j kSliceThreads + its number, four kSliceThreads further
    uint32_t keys[kSliceThreads], counts[kSliceWaves], firsts[kSliceWaves], down_to;
    double masses[kSliceWaves], powers[kPowers];
    unsigned long long bins[kMassBins];
};

__device__ inline void slice_row(const SampleProblem &p, uint32_t r, uint32_t slice, SliceShared &s)
{
    const LogitRow row(p, r);
    const RowParams q(p, r);
    const RowWork work(p, r);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), run = (work.units + kSliceWaves - 1) / kSliceWaves,
                   base = slice * work.units + wave * run, end = min(min(base + run, (slice + 1) * work.units), row.units()), from = base + lane;
    float mine = -INFINITY;
    {
        LogitRow::Raw raw[kSliceLoads];
#pragma unroll
        for (uint32_t j = 0; j < kSliceLoads; ++j)
            if (from + 64 * j < end) raw[j] = row.raw(from + 64 * j);
#pragma unroll
        for (uint32_t j = 0; j < kSliceLoads; ++j) {
            float x[8];
            if (from + 64 * j < end) row.convert(raw[j], from + 64 * j, x);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) mine = fmaxf(mine, x[i]);
            s.x[(2 * j) * kSliceThreads + threadIdx.x] = f32x4{x[0], x[1], x[2], x[3]};
            s.x[(2 * j + 1) * kSliceThreads + threadIdx.x] = f32x4{x[4], x[5], x[6], x[7]};
        }
    }
    s.keys[threadIdx.x] = key_of(mine);
    const bool massed = q.wants_mass(), limited = q.limited() && !q.greedy();
    const BinScale scale(q.temperature);
    const bool binned = massed && q.top_p < 1.0f && scale.usable();
    if (binned)
        for (uint32_t i = threadIdx.x; i < kMassBins; i += kSliceThreads) s.bins[i] = 0;
    if (massed && threadIdx.x < kPowers) s.powers[threadIdx.x] = SliceWeights::power(threadIdx.x);
    __syncthreads();
    // every wavefront has all of them
    const u32x4 key0 = *(const u32x4 *)&s.keys[4 * lane], key1 = *(const u32x4 *)&s.keys[256 + 4 * lane];
    const uint32_t key[8] = {key0[0], key0[1], key0[2], key0[3], key1[0], key1[1], key1[2], key1[3]};
    static_assert(kSliceThreads == 512, "eight a lane");
    uint32_t lane_key = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) lane_key = max(lane_key, key[i]);
    const float top = float_of(wave_largest(lane_key));
    const bool listed = limited && top != -INFINITY;
    if (listed && wave == 0) {
        // The lists' threshold, which at least `want` of the threads' largest logits reach, and at most a quarter more than that where a few steps
        // find such a one.  Each lane has eight of them: the smallest of the lanes' largest is reached by 64.
        const uint32_t want = q.top_k ? min(min((uint32_t)q.top_k, 2 * (uint32_t)q.top_k / work.slices + 32), 128u) : 64u;
        uint32_t down_to = want <= 64 ? ~wave_largest(~lane_key) : 0, above = key_of(top);
#pragma unroll 1
        for (int step = 0; step < 32 && above - down_to > 1; ++step) {
            const uint32_t to = down_to + (above - down_to) / 2;
            uint32_t reached = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) reached += __popcll(__ballot(key[i] >= to));
            if (reached < want) above = to;
            else {
                down_to = to;
                if (reached <= want + want / 4) break;
            }
        }
        // nothing that min_p keeps lies below this (the margin is for the roundings of this line; infinity has none: infinity less infinity is no number, whose place
        // among the keys its sign would decide)
        if (q.min_p > 0.0f && top != INFINITY) {
            const float below = q.temperature * logf(q.min_p);
            down_to = max(down_to, key_of(top + below - 1e-5f * (fabsf(top) + fabsf(below))));
        }
        if (lane == 0) s.down_to = max(down_to, key_of(-INFINITY) + 1);
    }
    if (limited) __syncthreads();
    const float low = listed ? float_of(s.down_to) : INFINITY;
    const bool has_top = __any(mine == top);
    const int32_t top_bin = scale.of(top);
    const SliceWeights weights(top, q.temperature, s.powers);
    Global<uint64_t> *list = work.list(slice, wave);
    uint32_t first = ~0u, count = 0;
    double mass = 0;
#pragma unroll 1
    for (uint32_t j = 0; j < kSliceLoads; ++j) {
        const f32x4 a = s.x[2 * j * kSliceThreads + threadIdx.x], b = s.x[(2 * j + 1) * kSliceThreads + threadIdx.x];
        const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        const uint32_t index = (from + 64 * j) * 8;
        if (has_top) {
#pragma unroll
            for (int i = 0; i < 8; ++i) first = x[i] == top ? min(first, index + i) : first;
        }
        if (listed) {
            uint32_t taken = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) taken |= (x[i] >= low ? 1u : 0u) << i;
            if (__any(taken != 0)) {
                const uint32_t up_to = count + wave_sum_scan((uint32_t)__popc(taken));
                uint32_t to = up_to - __popc(taken);
                count = lane_value(up_to, 63);
                if (count <= kListed)
                    while (taken) {
                        const uint32_t i = __builtin_ctz(taken);
                        taken &= taken - 1;
                        list[to++] = place_of(s.x[(2 * j + i / 4) * kSliceThreads + threadIdx.x][i % 4], index + i);
                    }
            }
        }
        if (massed && top != -INFINITY) {
#pragma unroll
            for (int half = 0; half < 8; half += 4) {
                double w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = top == INFINITY ? (x[half + i] == top ? 1.0 : 0.0) : weights.of(x[half + i]);
                mass += (w[0] + w[1]) + (w[2] + w[3]);
                if (binned) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t bin = (uint32_t)(top_bin - scale.of(x[half + i]));
                        // w + 2^8 is w in units, rounded, in front of the bits of 2^8
                        if (bin < kMassBins) atomicAdd(&s.bins[bin], (unsigned long long)(__builtin_bit_cast(uint64_t, w[i] + 256.0) - 0x4070000000000000ull));
                    }
                }
            }
        }
    }
    if (has_top) first = ~wave_largest(~first);
    if (massed) mass = wave_total(mass);
    if (lane == 0) {
        s.counts[wave] = count;
        s.firsts[wave] = first;
        s.masses[wave] = mass;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        Slice out{};
        uint32_t index = ~0u;
#pragma unroll
        for (uint32_t i = 0; i < kSliceWaves; ++i) {
            index = min(index, s.firsts[i]);
            out.mass += s.masses[i];
            out.count[i] = s.counts[i];
        }
        out.first = top == -INFINITY ? 0 : place_of(top, index);
        out.down_to = listed ? s.down_to : 0;
        out.bin = top_bin;
        out.binned = binned;
        work.store(slice, out);
    }
    if (binned)
        for (uint32_t i = threadIdx.x; i < kMassBins; i += kSliceThreads) work.bins(slice)[i] = s.bins[i];
}

template <typename Args>
__global__ __launch_bounds__(kSliceThreads, 8) void slice_rows(Args a)
{
    __shared__ SliceShared s;
    SampleProblem p;
    const uint32_t t = find_owner(a.first, a.p, a.base + blockIdx.x, p), slices = slices_of(p.V);
    slice_row(p, t / slices, t % slices, s);
}

// The code of this kernel runs once a row: what is not kept short is waited for line by line, so that loops are not unrolled and paths share their pieces.
constexpr uint32_t kPieceSums = 4;       // of a wavefront, 512 tokens each: a piece of a row has at most 2^19 / 16
struct ChooseShared {
    unsigned long long mass[kBins];
    uint32_t count[kBins];
    uint64_t places[kMostListed];
    uint64_t sums[kPieceSums * kSampleWaves];
    uint64_t part[kSampleWaves];
    double pieces[64];
    uint64_t before, prefix;
    uint32_t single, listed;
    int32_t token;
};

// Which of up to 64 pieces of a row (lane i: their kept weights, of the largest) has the token, and the weight in front of it there.
struct Piece { uint32_t at; double left; };
__device__ inline Piece choose_piece(const RowParams &q, double mass)
{
    const double all = wave_sum_scan(mass), target = q.before(lane_value(all, 63));
    // the first that passes the target, or the last that has any weight
    const uint64_t past = __ballot(all > target && mass > 0.0), any = __ballot(mass > 0.0);
    const uint32_t at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any | 1);
    return {at, target - (at ? lane_value(all, at - 1) : 0.0)};
}

// The token among logits from .. to of a row (from a multiple of eight), `left` (of the largest weight) in front of it there; `first` if nothing there weighs half a unit.
__device__ inline int32_t choose_in(const LogitRow &row, const RowLimits &l, uint32_t from, uint32_t to, double left, uint32_t first, ChooseShared &c)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, end = (to + 7) / 8;
    const auto eight = [&](uint32_t unit, uint64_t (&w)[8]) {
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 0;
        if (unit < end) {
            float x[8];
            row.convert(row.raw(unit), unit, x);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) sum += w[i] = l.kept(x[i], unit * 8 + i);
        }
        return sum;
    };
    __syncthreads();
    uint64_t w[8];
    uint32_t n = 0;
#pragma unroll 1
    for (uint32_t at = from / 8; at < end; at += kSampleThreads, ++n) {
        const uint64_t sum = wave_total(eight(at + threadIdx.x, w));
        if (lane == 0) c.sums[n * kSampleWaves + wave] = sum;
    }
    if (threadIdx.x == 0) c.token = (int32_t)first;
    __syncthreads();
    // sums of 64 units each: one wavefront finds whose token it is, and the token
    static_assert(kPieceSums * kSampleWaves == 64, "one a lane");
    if (wave == 0) {
        const uint64_t mine = lane < n * kSampleWaves ? c.sums[lane] : 0, scan = wave_sum_scan(mine), all = lane_value(scan, 63);
        if (all != 0) {
            // (the sums of pieces are rounded otherwise: the last token that weighs anything if none passes)
            const uint64_t want = min((uint64_t)(fmax(left, 0.0) * kWeightUnit), all - 1);
            const uint32_t owner = __builtin_ctzll(__ballot(scan > want)), unit = from / 8 + 64 * owner + lane;
            const uint64_t sum = eight(unit, w), up_to = lane_value(scan - mine, owner) + wave_sum_scan(sum);
            uint64_t before = up_to - sum;
            if (before <= want && want < up_to) {
                uint32_t at = 0;
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) {
                    if (before <= want) at = i;
                    before += w[i];
                }
                c.token = (int32_t)(unit * 8 + at);
            }
        }
    }
    __syncthreads();
    return c.token;
}

// The token of a row by reading all of it, once what is kept of it is known (l.cut, l.min_p): sixteen runs.
__device__ inline int32_t choose_by_runs(const LogitRow &row, const RowParams &q, const RowLimits &l, ChooseShared &c)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, run = (row.V + kSampleThreads - 1) / kSampleThreads * 64;
    const uint32_t from = wave * run, to = min(from + run, row.V);        // (the last ones may begin behind the row)
    uint64_t sum = 0;
#pragma unroll 1
    for (uint32_t unit = from / 8 + lane; unit < (to + 7) / 8; unit += 64) {
        float x[8];
        row.convert(row.raw(unit), unit, x);
#pragma unroll 2
        for (uint32_t i = 0; i < 8; ++i) sum += l.kept(x[i], unit * 8 + i);
    }
    sum = wave_total(sum);
    __syncthreads();
    if (lane == 0) c.part[wave] = sum;
    __syncthreads();
    const Piece piece = choose_piece(q, lane < kSampleWaves ? (double)c.part[lane] / kWeightUnit : 0.0);
    return choose_in(row, l, piece.at * run, min(piece.at * run + run, row.V), piece.left, index_of(l.first), c);
}

__device__ inline uint64_t block_total(uint64_t v, ChooseShared &c)
{
    v = wave_total(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) c.part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t all = 0;
    for (uint32_t i = 0; i < kSampleWaves; ++i) all += c.part[i];
    return all;
}

// The place of the token with which the first ones of an order reach `target`, tokens or weight, among those whose places begin with `prefix` in front of the last
// `left` bits.  each(f) calls f for each of a thread's tokens.  What it gives is at most that place, and above that of the next token of these.
template <typename Each>
__device__ inline uint64_t reach(const Each &each, const RowLimits &l, bool by_weight, uint64_t target, uint64_t prefix, uint32_t left, ChooseShared &c)
{
    for (;;) {
        const uint32_t bits = min(left, 11u), rest = left - bits;
        for (uint32_t i = threadIdx.x; i < kBins; i += kSampleThreads) {
            c.mass[i] = 0;
            c.count[i] = 0;
        }
        __syncthreads();
        each([&](uint64_t place) {
            if (left < kPlaceBits && place >> left != prefix) return;
            const uint32_t bin = kBins - 1 - ((uint32_t)(place >> rest) & ((1u << bits) - 1));
            atomicAdd(&c.count[bin], 1u);
            if (by_weight) atomicAdd(&c.mass[bin], (unsigned long long)l.units(l.of(logit_of(place))));
        });
        __syncthreads();
        // two bins a thread, the earliest tokens in front
        const uint32_t b = 2 * threadIdx.x;
        const uint64_t n0 = by_weight ? c.mass[b] : c.count[b], n1 = by_weight ? c.mass[b + 1] : c.count[b + 1];
        const uint64_t up_to = wave_sum_scan(n0 + n1);
        uint64_t before = up_to - (n0 + n1);
        if ((threadIdx.x & 63) == 63) c.part[threadIdx.x >> 6] = up_to;
        __syncthreads();
        for (uint32_t i = 0; i < threadIdx.x >> 6; ++i) before += c.part[i];
        const bool one = before < target && target <= before + n0, two = before + n0 < target && target <= before + n0 + n1;
        if (one || two) {
            const uint32_t bin = b + two;
            c.before = before + (two ? n0 : 0);
            c.prefix = (left < kPlaceBits ? prefix << bits : 0) | ((kBins - 1 - bin) & ((1u << bits) - 1));
            c.single = c.count[bin] == 1;
        }
        __syncthreads();
        prefix = c.prefix;
        target -= c.before;
        left = rest;
        const bool done = c.single || left == 0;
        __syncthreads();
        if (done) return prefix << left;
    }
}

// Among the row's tokens down to l.cut.
__device__ inline uint64_t reach_in_row(const LogitRow &row, const RowLimits &l, bool by_weight, uint64_t target, ChooseShared &c)
{
    return reach([&](const auto &f) {
#pragma unroll 1
        for (uint32_t i = threadIdx.x; i < row.V; i += kSampleThreads) {
            const float x = row[i];
            const uint64_t place = place_of(x, i);
            if (x != -INFINITY && place >= l.cut) f(place);
        }
    }, l, by_weight, target, 0, kPlaceBits, c);
}

// The token of a row by reading it as often as it takes; l.cut is 0.
__device__ inline int32_t choose_anywhere(const LogitRow &row, const RowParams &q, RowLimits &l, ChooseShared &c)
{
    __syncthreads();
    if (q.top_k) {
        // logits of minus infinity have no place: fewer may be left
        uint64_t count = 0;
        for (uint32_t i = threadIdx.x; i < row.V; i += kSampleThreads) count += row[i] != -INFINITY;
        count = block_total(count, c);
        if ((uint32_t)q.top_k < count) l.cut = reach_in_row(row, l, false, (uint32_t)q.top_k, c);
    }
    if (q.top_p < 1.0f) {
        uint64_t total = 0;
        for (uint32_t i = threadIdx.x; i < row.V; i += kSampleThreads) {
            const float x = row[i];
            total += x != -INFINITY && place_of(x, i) >= l.cut ? l.units(l.of(x)) : 0;
        }
        total = block_total(total, c);
        l.cut = max(l.cut, reach_in_row(row, l, true, min(q.share((double)total), total), c));
    }
    return choose_by_runs(row, q, l, c);
}

// The lists of a row's slices, one behind the other, so in order of index; how many, more than kMostListed if they do not fit.
__device__ inline uint32_t gather_lists(const RowWork &work, const Slice &mine, ChooseShared &c)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t most = 0, own = 0;
#pragma unroll
    for (uint32_t v = 0; v < kSliceWaves; ++v) {
        most = max(most, mine.count[v]);
        own = min(own + mine.count[v], kMostListed + 1);
    }
    const uint32_t scan = wave_sum_scan(own), all = lane_value(scan, 63);
    if (__any(most > kListed) || all > kMostListed) return kMostListed + 1;
    // where each list goes
    if (wave == 0 && lane < work.slices) {
        uint32_t to = scan - own;
#pragma unroll
        for (uint32_t v = 0; v < kSliceWaves; ++v) {
            c.count[lane * kSliceWaves + v] = to;
            to += mine.count[v];
            c.count[1024 + lane * kSliceWaves + v] = to;
        }
    }
    __syncthreads();
    static_assert(kListed == 64 && kSliceWaves * 64 <= 1024, "one a lane");
    const Global<uint64_t> *lists = work.list(0, 0);
    // eight lists of a wavefront at once; what stands behind a list's end is read and dropped
#pragma unroll 1
    for (uint32_t i0 = wave; i0 < work.slices * kSliceWaves; i0 += 8 * kSampleWaves) {
        uint64_t place[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) place[k] = lists[min(i0 + k * kSampleWaves, work.slices * kSliceWaves - 1) * kListed + lane];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
            const uint32_t i = i0 + k * kSampleWaves;
            if (i >= work.slices * kSliceWaves) break;
            const uint32_t to = c.count[i] + lane;
            if (to < c.count[1024 + i]) c.places[to] = place[k];
        }
    }
    __syncthreads();
    return all;
}

// The token of a row whose lists have what its limits may keep: known down to `down_to` (the upper bits of a place).  total: the row's weight, if it is known.  -1 if the lists
// do not tell.  (By one wavefront alone, without barriers, 256 rows with top_k 200 took 22 us, with this 16; with top_k 50 both 16.)
__device__ inline int32_t choose_listed(uint32_t count, const RowParams &q, RowLimits l, uint32_t down_to, double total, ChooseShared &c)
{
    static_assert(kMostListed == 4 * kSampleThreads, "four places a thread");
    const double min_p = l.min_p;
    l.min_p = 0;             // (for the sums)
    // everything there is is known, or everything that min_p keeps
    const bool everything = down_to <= key_of(-INFINITY) + 1;
    bool known = everything || (min_p > 0.0 && l.of(float_of(down_to)) < min_p);
    uint64_t cut = (uint64_t)down_to << 20;
    const auto each = [&](const auto &f) {
#pragma unroll 1
        for (uint32_t j = threadIdx.x; j < count; j += kSampleThreads)
            if (c.places[j] >= cut) f(c.places[j]);
    };
    // what lies between `cut` and the first token
    const auto reach_from_cut = [&](bool by_weight, uint64_t target) {
        const uint32_t left = l.first == cut ? 0 : 64 - __builtin_clzll(l.first ^ cut);
        cut = left == 0 ? cut : max(cut, reach(each, l, by_weight, target, l.first >> left, left, c));
    };
    if (q.top_k) {
        uint64_t n = 0;
        each([&](uint64_t) { ++n; });
        n = block_total(n, c);
        if (n >= (uint32_t)q.top_k) known = true;
        else if (!everything && q.top_p < 1.0f) return -1;         // the sum of what top_k keeps is not known
        if (n > (uint32_t)q.top_k) reach_from_cut(false, (uint32_t)q.top_k);
    }
    if (q.top_p < 1.0f) {
        uint64_t weight = 0;
        each([&](uint64_t place) { weight += l.units(l.of(logit_of(place))); });
        weight = block_total(weight, c);
        const bool all = everything || q.top_k;      // these are all that share the weight
        const uint64_t target = all ? min(q.share((double)weight), weight) : q.share(total);
        if (target <= weight) {
            known = true;
            reach_from_cut(true, target);
        }
    }
    if (!known) return -1;
    l.min_p = min_p;
    uint64_t w[4], sum = 0;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
        const uint32_t j = 4 * threadIdx.x + k;
        const uint64_t place = j < count ? c.places[j] : 0;
        w[k] = j < count && place >= cut ? l.kept(logit_of(place), index_of(place)) : 0;
        sum += w[k];
    }
    const uint64_t scan = wave_sum_scan(sum);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) c.part[threadIdx.x >> 6] = scan;
    __syncthreads();
    uint64_t before = scan - sum, all = 0;
#pragma unroll
    for (uint32_t i = 0; i < kSampleWaves; ++i) {
        before += i < threadIdx.x >> 6 ? c.part[i] : 0;
        all += c.part[i];
    }
    const uint64_t want = min((uint64_t)q.before((double)all), all - 1);      // (the product may be rounded up)
    if (before <= want && want < before + sum) {
        uint32_t k = 0;
        while (k < 3 && before + w[k] <= want) before += w[k++];
        c.token = (int32_t)index_of(c.places[4 * threadIdx.x + k]);
    }
    __syncthreads();
    return c.token;
}

// The bin in which the row's weight reaches `share` units (lane i: slice i), by all slices' bins, and how much of it that takes; false if it is none of theirs.
// front: lane i gets slice i's weight in front of it.
struct LastBin { int32_t bin; double want, front; };
__device__ inline bool find_bin(const RowWork &work, const RowLimits &l, const Slice &mine, int32_t top_bin, double share, LastBin &last, ChooseShared &c)
{
    static_assert(kMassBins <= kSampleThreads && kMassBins % 64 == 0, "a bin a thread");
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double factor = mine.first ? l.of(logit_of(mine.first)) : 0.0;
    if (__any(lane < work.slices && mine.first && !mine.binned)) return false;
    double sum = 0;
    if (threadIdx.x < kMassBins) {
#pragma unroll 1
        for (uint32_t i0 = 0; i0 < work.slices; i0 += 8) {
            uint64_t v[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) {
                const uint32_t i = min(i0 + k, work.slices - 1), bin = threadIdx.x - (uint32_t)(top_bin - lane_value(mine.bin, i));
                v[k] = 0;
                if (i0 + k < work.slices && lane_value(factor, i) > 0.0 && bin < kMassBins) v[k] = work.bins(i)[bin];
            }
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) sum = fma((double)v[k], lane_value(factor, min(i0 + k, work.slices - 1)), sum);
        }
    }
    double *part = (double *)c.part;
    const double up_to = wave_sum_scan(sum);
    __syncthreads();
    if (threadIdx.x == 0) c.single = 0;
    if (lane == 63) part[wave] = up_to;
    __syncthreads();
    double before = 0;
    for (uint32_t i = 0; i < wave; ++i) before += part[i];
    // the first bin that reaches it: sums rounded differently may leave none or two at a border of wavefronts, of which none is taken
    if (threadIdx.x < kMassBins && before + (up_to - sum) < share && share <= before + up_to && atomicAdd(&c.single, 1u) == 0) {
        c.before = __builtin_bit_cast(uint64_t, share - (before + (up_to - sum)));
        c.prefix = (uint64_t)(int64_t)(top_bin - (int32_t)threadIdx.x);
    }
    __syncthreads();
    last.want = __builtin_bit_cast(double, c.before);
    last.bin = (int32_t)c.prefix;
    if (c.single != 1) return false;
#pragma unroll 1
    for (uint32_t i = wave; i < work.slices; i += kSampleWaves) {
        const int32_t bins = lane_value(mine.bin, i) - last.bin;       // of this slice in front of the last
        const double f = lane_value(factor, i);
        uint64_t v = 0;
#pragma unroll
        for (uint32_t k = 0; k < kMassBins / 64; ++k)
            if (f > 0.0 && (int32_t)(lane + 64 * k) < bins) v += work.bins(i)[lane + 64 * k];
        const uint64_t all = wave_total(v);
        if (lane == 0) c.pieces[i] = (double)all / kWeightUnit * f;
    }
    __syncthreads();
    last.front = lane < work.slices ? c.pieces[lane] : 0.0;
    return true;
}

// Finds the last kept place (l.cut) in the bin in which top_p ends: reads the row for the bin's tokens; false if they are too many.
__device__ inline bool cut_in_bin(const LogitRow &row, const RowParams &q, RowLimits &l, const LastBin &last, ChooseShared &c)
{
    constexpr uint32_t kAtOnce = 4;
    const uint32_t lane = threadIdx.x & 63, units = row.units();
    // the bin's logits: bins do not fall as logits grow, so a search among the floats' numbers finds its smallest and the next bin's
    const BinScale scale(q.temperature);
    const auto first_of = [&](int32_t bin) {
        uint32_t low = key_of(-INFINITY), high = key_of(INFINITY);       // the bin of `low` is smaller; `high` is that of infinity
#pragma unroll 1
        while (high - low > 1) {
            const uint32_t step = (high - low + 63) / 64, at = min(low + (lane + 1) * step, high);
            const uint32_t reached = __builtin_ctzll(__ballot(at == high || scale.of(float_of(at)) >= bin));
            high = min(low + (reached + 1) * step, high);
            low += reached * step;
        }
        return high;
    };
    const uint32_t low = first_of(last.bin), high = first_of(last.bin + 1);
    if (low >= high) return false;
    const float from = float_of(low), to = float_of(high - 1);
    if (threadIdx.x == 0) c.listed = 0;
    __syncthreads();
#pragma unroll 1
    for (uint32_t unit = threadIdx.x; unit < units; unit += kAtOnce * kSampleThreads) {
        LogitRow::Raw raw[kAtOnce];
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k)
            if (unit + k * kSampleThreads < units) raw[k] = row.raw(unit + k * kSampleThreads);
        float x[kAtOnce][8];
        uint32_t marked = 0;
#pragma unroll
        for (uint32_t k = 0; k < kAtOnce; ++k) {
            if (unit + k * kSampleThreads >= units) break;
            row.values(raw[k], x[k]);
            uint32_t among = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) among |= (__builtin_amdgcn_fmed3f(x[k][i], from, to) == x[k][i] ? 1u : 0u) << i;      // (no NaN is)
            if ((unit + k * kSampleThreads) * 8 + 8 > row.V) among &= (1u << row.V % 8) - 1;
            marked |= among << (8 * k);
        }
        // one for all of a thread's: what waits costs more than what is counted
        uint32_t slot = marked ? atomicAdd(&c.listed, (uint32_t)__popc(marked)) : 0;
        while (marked) {
            const uint32_t at = __builtin_ctz(marked);
            float value = x[0][0];
#pragma unroll
            for (uint32_t j = 1; j < 8 * kAtOnce; ++j) value = at == j ? x[j / 8][j % 8] : value;
            marked &= marked - 1;
            if (slot < kMostListed) c.places[slot] = place_of(LogitRow::clean(value), (unit + at / 8 * kSampleThreads) * 8 + at % 8);
            ++slot;
        }
    }
    __syncthreads();
    const uint32_t count = c.listed;
    if (count > kMostListed) return false;
    // the bin's weight, and what its places have in common
    uint64_t weight = 0, most = 0, least = 0;
    const auto each = [&](const auto &f) {
#pragma unroll 1
        for (uint32_t j = threadIdx.x; j < count; j += kSampleThreads) f(c.places[j]);
    };
    each([&](uint64_t place) {
        most = max(most, place);
        least = max(least, ~place);
        weight += l.units(l.of(logit_of(place)));
    });
    weight = block_total(weight, c);
    if (weight == 0) return false;
    most = wave_largest(most);
    least = wave_largest(least);
    if (threadIdx.x == 0) c.before = c.prefix = 0;
    __syncthreads();
    if (lane == 0) {
        atomicMax((unsigned long long *)&c.before, (unsigned long long)most);
        atomicMax((unsigned long long *)&c.prefix, (unsigned long long)least);
    }
    __syncthreads();
    most = c.before;
    const uint64_t smallest = ~c.prefix;
    const uint32_t left = most == smallest ? 0 : 64 - __builtin_clzll(most ^ smallest);
    __syncthreads();
    // (not below the bin: what lies there is none of `each`)
    l.cut = left == 0 ? most : max(smallest, reach(each, l, true, min(max((uint64_t)ceil(last.want), (uint64_t)1), weight), most >> left, left, c));
    return true;
}

__device__ inline int32_t choose_row(const SampleProblem &p, uint32_t r, ChooseShared &c)
{
    const LogitRow row(p, r);
    const uint32_t lane = threadIdx.x & 63;
    const RowWork work(p, r);
    // lane i of every wavefront has slice i
    Slice mine{};
    if (lane < work.slices) mine = work.load(lane);
    const RowParams q(p, r);
    const uint64_t first = wave_largest(mine.first);
    if (first == 0) return -1;
    if (q.greedy()) return (int32_t)index_of(first);
    RowLimits l(first, q.temperature, q.min_p);
    double mass = mine.first && q.wants_mass() ? mine.mass * l.of(logit_of(mine.first)) : 0.0;
    if (q.limited()) {
        const double total = wave_total(mass) * kWeightUnit;
        const uint32_t count = gather_lists(work, mine, c);
        if (count <= kMostListed) {
            const uint32_t down_to = wave_largest(lane < work.slices && mine.first ? mine.down_to : 0);
            const int32_t token = choose_listed(count, q, l, down_to, total, c);
            if (token >= 0) return token;
        }
        LastBin last;
        const bool by_bin = !q.top_k && q.top_p < 1.0f && find_bin(work, l, mine, BinScale(q.temperature).of(l.top), (double)q.share(total), last, c) && cut_in_bin(row, q, l, last, c);
        if (!by_bin) {
            l.cut = 0;
            if (q.top_k || q.top_p < 1.0f) return choose_anywhere(row, q, l, c);
        }
        if (q.min_p > 0.0f) return choose_by_runs(row, q, l, c);
        // what is kept of the bin goes to the slices; the histogram's place holds their sums
        __syncthreads();
        if (threadIdx.x < 64) c.mass[threadIdx.x] = 0;
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < c.listed; j += kSampleThreads) {
            const uint32_t index = index_of(c.places[j]);
            const uint64_t w = l.kept(logit_of(c.places[j]), index);
            if (w) atomicAdd(&c.mass[index / 8 / work.units], (unsigned long long)w);
        }
        __syncthreads();
        mass = last.front + (double)c.mass[lane] / kWeightUnit;
    }
    const Piece piece = choose_piece(q, mass);
    const uint32_t from = piece.at * work.units * 8;
    return choose_in(row, l, from, min(from + work.units * 8, row.V), piece.left, index_of(lane_value(mine.first, piece.at)), c);
}

template <typename Args>
__global__ __launch_bounds__(kSampleThreads) void choose_rows(Args a)
{
    __shared__ ChooseShared s;
    SampleProblem p;
    const uint32_t r = find_owner(a.first, a.p, a.base + blockIdx.x, p);
    const int32_t token = choose_row(p, r, s);
    if (threadIdx.x == 0) ((Global<int32_t> *)p.tokens)[r] = token;
}

uint64_t sample_work_bytes(uint32_t M, uint32_t V) { return M * RowWork::size(V); }

namespace {

template <uint32_t NP>
hipError_t launch_sampling(const SampleProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    hipError_t e = launch_answer_of<SampleProblem, NP>(slice_rows, kSliceThreads, p, n, stream, launches, [](const SampleProblem &q) { return (uint64_t)q.M * slices_of(q.V); });
    if (e == hipSuccess) e = launch_answer_of<SampleProblem, NP>(choose_rows, kSampleThreads, p, n, stream, launches, [](const SampleProblem &q) { return (uint64_t)q.M; });
    return e;
}

}  // namespace

hipError_t launch_sample(const SampleProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    return n <= kAnswerFew ? launch_sampling<kAnswerFew>(p, n, stream, launches) : launch_sampling<kAnswerProblems>(p, n, stream, launches);
}

}  // namespace salus
