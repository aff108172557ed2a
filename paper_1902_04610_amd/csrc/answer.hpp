// What the kernels of answering models share: a job's sequences and their paged cache as the kernels see them, the lookup workgroup -> (job, sequence, tile), and
// the launchers.
#pragma once
#include "block.hpp"

namespace salus {

// New rows of a job, the sequences they belong to and the cache behind them (the arrays are the caller's device memory: whatever they
// hold, nothing outside is touched).
struct Sequences {
    const int32_t *starts, *lens, *table;
    uint32_t n_seqs, M, max_pages, n_pages;
    uint32_t Hq, Hkv, D;
    uint32_t page_bits;      // log2 of the tokens of a page
};

struct AppendProblem {
    Sequences seq;
    const void *x;
    void *q, *k, *v;
    const double *freq;
    uint32_t rotary, interleaved;
    float magnitude;
    uint32_t pad;
};
hipError_t launch_append(const AppendProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches);

struct AttentionProblem {
    Sequences seq;
    const void *q, *k, *v;
    void *y;
    float *work;             // sums of the parts of a row's keys
    uint32_t max_len, window;
    float scale;             // times log2(e)
    uint32_t part;           // keys of a part, a multiple of 128
    uint32_t parts;          // of a row at most
    uint32_t columns;        // of a tile
};
struct AttentionParts { uint32_t columns, part, parts; };
AttentionParts attention_parts(uint32_t M, uint32_t n_seqs, uint32_t Hq, uint32_t Hkv, uint32_t D, uint32_t max_len, uint32_t window);
uint64_t attention_work_floats(uint32_t M, uint32_t Hq, uint32_t D, const AttentionParts &);      // that a call uses
uint64_t attention_room_floats(uint32_t M, uint32_t Hq, uint32_t Hkv, uint32_t D, uint32_t max_len);      // at least that of calls of up to M rows and max_len tokens
hipError_t launch_attention(const AttentionProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches);

struct SampleProblem {
    const void *logits;
    const uint32_t *params;      // M x {temperature, top_k, top_p, min_p}
    const float *u;
    int32_t *tokens;
    void *work;
    uint32_t M, V, ld, bf16;
};
uint64_t sample_work_bytes(uint32_t M, uint32_t V);
hipError_t launch_sample(const SampleProblem *p, uint32_t n, hipStream_t stream, uint64_t *launches);

// Launches by value of at most 24 problems, or of at most 4 for rounds whose time is the host's.
template <typename P, uint32_t NP>
struct AnswerArgs {
    uint32_t n, tiles, base, pad;
    uint32_t first[NP];      // first tile of problem i; kNoTile from n on
    P p[NP];
};
constexpr uint32_t kAnswerFew = 4;
constexpr uint32_t kAnswerProblems = 24;
static_assert(sizeof(AnswerArgs<AppendProblem, kAnswerProblems>) <= 4096 && sizeof(AnswerArgs<AttentionProblem, kAnswerProblems>) <= 4096,
              "kernel arguments are limited to 4 KB");

// Runs n problems through launches of as many as fit, by their arguments and by their tiles, which have 31-bit numbers: kernel(args) of `threads` threads a workgroup, one for
// each of tiles(problem).
template <typename P, uint32_t NP, typename Tiles>
inline hipError_t launch_answer_of(void (*kernel)(AnswerArgs<P, NP>), int threads, const P *p, uint32_t n, hipStream_t stream, uint64_t *launches, Tiles tiles)
{
    for (uint32_t at = 0, count = 0; at < n; at += count) {
        AnswerArgs<P, NP> a{};
        count = n - at < NP ? n - at : NP;
        uint64_t total;
        while ((total = fill_group(a, p + at, count, tiles)) > 0x7fffffffull) {
            if (count == 1) return hipErrorInvalidValue;
            count = (count + 1) / 2;
        }
        const hipError_t e = launch_tiles(total, threads, launches, [&](uint32_t blocks, uint32_t base) {
            a.base = base;
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, stream, a);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// A tile of a sequence's rows.
struct SequenceTile {
    uint32_t s, row, n;      // the sequence, its first row, its rows
    uint32_t tile;           // number of the tile among those of the sequence
    int32_t length;          // its tokens
};

// Tiles are numbered so that none has to be counted: sequence s begins at tile base(start of s, s), which leaves it as many as it can need, and
// some that stay empty.  Sixty-four sequences are looked at at once, their beginnings, ends and lengths, so that the search is one trip to memory for up to 64
// of them, two for 4096.  length: at most `most`.
template <typename Base>
__device__ inline bool find_sequence(const Sequences &q, uint32_t t, Base base, uint32_t most, SequenceTile &out)
{
    const uint32_t lane = threadIdx.x & 63;
    const Global<int32_t> *starts = (const Global<int32_t> *)q.starts, *lens = (const Global<int32_t> *)q.lens;
    const auto row = [&](int32_t v) { return (uint32_t)min(max(v, 0), (int32_t)q.M); };
    uint32_t low = 0, span = q.n_seqs;
    for (;;) {
        const uint32_t step = (span + 63) / 64, s = min(low + lane * step, q.n_seqs - 1);
        const uint32_t start = row(starts[s]), end = row(starts[s + 1]), length = (uint32_t)min(max(lens[s], 0), (int32_t)most);
        const uint64_t before = __ballot(lane * step < span && base(start, s) <= t);
        if (before == 0) return false;
        const uint32_t at = 63 - __builtin_clzll(before);
        low += at * step;
        span = min(step, span - at * step);
        if (span > 1) continue;
        const uint32_t first = lane_value(start, at), behind = lane_value(end, at);
        out = {low, first, behind > first ? behind - first : 0, t - base(first, low), (int32_t)lane_value(length, at)};
        return true;
    }
}

}  // namespace salus
