// Appends to the paged caches of a round's jobs: queries and keys of the new rows are rotated by their positions, keys and values go to their places.
//
//   pair (a, b) of frequency f at position p:   a cos(p f) - b sin(p f),  a sin(p f) + b cos(p f),  times the magnitude
//
// Bound by memory where there are many rows: every element is read once and written once.  A workgroup takes the new tokens of one aligned group of eight of a
// sequence, because eight tokens are what lies together in the cache: a key's eight elements of eight tokens are a line, as are a value
// element's of eight tokens times eight elements.  Cosines and sines of the eight positions are made once for all heads, in 64 bits (a
// position of 10^6 times a frequency of 1 is off by 0.03 rad in 32) and kept as floats in LDS.  A thread asks for four
// units before it turns any: 110 us for 514 MB of prompts (121 one by one; asking before the cosines, or for five, gains nothing).
#include "answer.hpp"

namespace salus {

constexpr uint32_t kAppendThreads = 256, kMostPairs = 128, kAtOnce = 4;

// Tiles of a sequence: its groups of eight tokens, which begin anywhere; at most (n + 7) / 8 + 1 of them.
__host__ __device__ inline uint32_t append_base(uint32_t start, uint32_t s) { return start / 8 + 2 * s; }

// Elements d .. d + 7 of a head and, where each has its partner in one other unit, that unit.
struct Unit {
    const Global<char> *head;
    uint32_t d;
    u32x4 own, other;
    __device__ void load(const Global<char> *h, uint32_t at, uint32_t rotary, uint32_t interleaved)
    {
        head = h;
        d = at;
        own = *(const Global<u32x4> *)(head + 2 * d);
        if (!interleaved && rotary % 16 == 0) other = d < rotary ? *(const Global<u32x4> *)(head + 2 * (d < rotary / 2 ? d + rotary / 2 : d - rotary / 2)) : own;
    }
};

// Rotated in the first `rotary` elements of a head, with cs the cosines and sines of the pairs.
__device__ inline u32x4 rotate8(const Unit &unit, uint32_t rotary, uint32_t interleaved, const float2 *cs)
{
    const u32x4 own = unit.own, other = unit.other;
    const uint32_t d = unit.d;
    if (d >= rotary) return own;
    float e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[2 * i] = bf16_low(own[i]);
        e[2 * i + 1] = bf16_high(own[i]);
    }
    float r[8];
    const uint32_t half = rotary / 2;
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = cs[min(d / 2 + i, half - 1)];
            const bool in = d + 2 * i < rotary;
            r[2 * i] = in ? e[2 * i] * t.x - e[2 * i + 1] * t.y : e[2 * i];
            r[2 * i + 1] = in ? e[2 * i] * t.y + e[2 * i + 1] * t.x : e[2 * i + 1];
        }
    } else {
        float o[8];
        if (half % 8 == 0) {         // the partners are a unit of their own
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[2 * i] = bf16_low(other[i]);
                o[2 * i + 1] = bf16_high(other[i]);
            }
        } else {                     // each by itself: 201 us for 24000 rows of 32 heads of 128 on 8, rotary 122, where 128 takes 142
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t at = d + i < half ? d + i + half : d + i < rotary ? d + i - half : d + i;
                o[i] = bf16_low(((const Global<uint16_t> *)unit.head)[at]);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t at = d + i;
            const float2 t = cs[min(at < half ? at : at - half, half - 1)];
            r[i] = at >= rotary ? e[i] : at < half ? e[i] * t.x - o[i] * t.y : o[i] * t.y + e[i] * t.x;
        }
    }
    return {bf16_pack(r[0], r[1]), bf16_pack(r[2], r[3]), bf16_pack(r[4], r[5]), bf16_pack(r[6], r[7])};
}

template <typename Args>
__global__ __launch_bounds__(kAppendThreads) void append_rows(Args a)
{
    __shared__ float2 cs[8][kMostPairs];
    AppendProblem p;
    const uint32_t t = find_owner(a.first, a.p, a.base + blockIdx.x, p);
    SequenceTile at;
    // a sequence may be longer than what max_pages hold: its tokens there have no page
    if (!find_sequence(p.seq, t, append_base, 0x7fffff00, at)) return;
    const Sequences &s = p.seq;
    const int32_t position = at.length - (int32_t)at.n;          // of the sequence's first new row
    const int32_t group = (position & ~7) + 8 * (int32_t)at.tile;                     // first token of the eight
    const int32_t from = max(group, position), to = min(group + 8, position + (int32_t)at.n);
    if (from >= to) return;
    const uint32_t count = to - from, pairs = p.rotary / 2;
    const uint64_t row = (uint64_t)at.row + (from - position);
    for (uint32_t i = threadIdx.x; i < count * pairs; i += kAppendThreads) {
        const uint32_t j = i / pairs, f = i % pairs;
        double sine, cosine;
        sincos((double)(from + (int32_t)j) * ((const Global<double> *)p.freq)[f], &sine, &cosine);
        cs[j][f] = {(float)(cosine * p.magnitude), (float)(sine * p.magnitude)};
    }
    __syncthreads();

    const uint32_t units = s.D / 8, heads = s.Hq + s.Hkv, pitch = (s.Hq + 2 * s.Hkv) * s.D;
    const Global<char> *x = (const Global<char> *)p.x + row * pitch * 2;
    // the page of the eight (they never straddle two), and where its keys and values of head 0 begin
    const uint32_t page_of = (uint32_t)max(group, 0) >> s.page_bits, slot = (uint32_t)max(group, 0) & ((1u << s.page_bits) - 1);
    const int32_t page = group >= 0 && page_of < s.max_pages ? ((const Global<int32_t> *)s.table)[(uint64_t)at.s * s.max_pages + page_of] : -1;
    const bool stored = page >= 0 && (uint32_t)page < s.n_pages;
    const uint64_t head_bytes = (uint64_t)(2 * s.D) << s.page_bits, block = (uint64_t)(stored ? page : 0) * s.Hkv * head_bytes;
    const uint32_t lead = from - group;                  // tokens of the eight in front of the first

    // eight tokens: lanes of a wavefront take eight units of eight tokens, lines on both sides; fewer: units of one token after the other
    const uint32_t tokens = count == 8 ? 8 : 1, each = heads * units * tokens;
    for (uint32_t j0 = 0; j0 < count; j0 += tokens)
        for (uint32_t i0 = threadIdx.x; i0 < each; i0 += kAtOnce * kAppendThreads) {
            const auto place = [&](uint32_t i, uint32_t &j, uint32_t &h, uint32_t &d) {
                const uint32_t at = min(i, each - 1), unit = at / tokens;
                j = j0 + at % tokens;
                h = unit / units;
                d = unit % units * 8;
            };
            Unit asked[kAtOnce];
#pragma unroll
            for (uint32_t k = 0; k < kAtOnce; ++k) {
                uint32_t j, h, d;
                place(i0 + k * kAppendThreads, j, h, d);
                asked[k].load(x + ((uint64_t)j * pitch + h * s.D) * 2, d, p.rotary, p.interleaved);
            }
#pragma unroll
            for (uint32_t k = 0; k < kAtOnce; ++k) {
                if (i0 + k * kAppendThreads >= each) break;
                uint32_t j, h, d;
                place(i0 + k * kAppendThreads, j, h, d);
                const u32x4 w = rotate8(asked[k], p.rotary, p.interleaved, cs[j]);
                if (h < s.Hq) *(Global<u32x4> *)((Global<char> *)p.q + ((row + j) * s.Hq + h) * (uint64_t)(s.D * 2) + d * 2) = w;
                else if (stored) {
                    const uint32_t token = slot + lead + j;
                    *(Global<u32x4> *)((Global<char> *)p.k + block + (h - s.Hq) * head_bytes + (uint64_t)(token / 32 * (s.D / 8) + d / 8) * 512 + token % 32 * 16) = w;
                }
            }
        }
    if (!stored) return;
    const Global<char> *values = x + (uint64_t)heads * s.D * 2;
    for (uint32_t i = threadIdx.x; i < s.Hkv * s.D / 2; i += kAppendThreads) {
        const uint32_t h = i / (s.D / 2), d = i % (s.D / 2) * 2;
        Global<char> *to_v = (Global<char> *)p.v + block + h * head_bytes + (uint64_t)(slot / 8 * s.D + d) * 16;
        const Global<char> *from_v = values + (h * s.D + d) * 2;
        if (count == 8) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = *(const Global<uint32_t> *)(from_v + (uint64_t)j * pitch * 2);
            u32x4 low, high;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                low[j] = (w[2 * j] & 0xffffu) | w[2 * j + 1] << 16;
                high[j] = w[2 * j] >> 16 | (w[2 * j + 1] & 0xffff0000u);
            }
            *(Global<u32x4> *)to_v = low;
            *(Global<u32x4> *)(to_v + 16) = high;
        } else {
            for (uint32_t j = 0; j < count; ++j) {
                const uint32_t w = *(const Global<uint32_t> *)(from_v + (uint64_t)j * pitch * 2);
                ((Global<uint16_t> *)to_v)[lead + j] = (uint16_t)w;
                ((Global<uint16_t> *)(to_v + 16))[lead + j] = (uint16_t)(w >> 16);
            }
        }
    }
}

hipError_t launch_append(const AppendProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches)
{
    const auto tiles = [](const AppendProblem &q) { return (uint64_t)append_base(q.seq.M, q.seq.n_seqs); };
    if (n <= kAnswerFew) return launch_answer_of<AppendProblem, kAnswerFew>(append_rows, kAppendThreads, p, n, stream, launches, tiles);
    return launch_answer_of<AppendProblem, kAnswerProblems>(append_rows, kAppendThreads, p, n, stream, launches, tiles);
}

}  // namespace salus
