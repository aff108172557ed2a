// What the attention kernels share: which rows and keys a workgroup has, softmax weights of a tile of scores, values that are no numbers.
//
// A column is one (row, query head) of a sequence and a key head; the columns of a key head follow each other row by row, its query heads fastest, so that heads
// that share keys fill a tile.  S^T = K Q^T puts a column into one lane of each group of lanes, and with them its scores; these are, rounded to bf16, the second
// operand of O^T = V^T P^T as they are: the contraction runs over keys in any order as long as V's is the same, and K's rows are taken in the
// order that gives a lane the eight consecutive keys whose values lie together in the cache.  Scores and weights never pass through LDS: attend_few has the join of its wavefronts there,
// attend_many the keys and values that its wavefronts share.
#pragma once
#include "answer.hpp"

namespace salus {

constexpr uint32_t kKeys = 32;      // of a tile

// Tiles of `columns` columns of a sequence: G query heads share a key head.
struct ColumnBase {
    uint32_t G, columns;
    __host__ __device__ uint32_t operator()(uint32_t start, uint32_t s) const { return start * G / columns + s; }
};
inline uint64_t column_tiles(const AttentionProblem &q)
{
    return (uint64_t)ColumnBase{q.seq.Hq / q.seq.Hkv, q.columns}(q.seq.M, q.seq.n_seqs) * q.seq.Hkv;
}

// A window, cut so that positions and windows can be subtracted.
__device__ inline int32_t window_of(const AttentionProblem &p) { return (int32_t)min(p.window, 1u << 30); }

// A tile of columns: which rows, and which keys any of them sees.
struct ColumnTile {
    uint32_t head;              // key head
    uint32_t s, row, n;         // the sequence, its first row, its rows
    uint32_t first, end;        // columns of the tile among the sequence's
    int32_t position;           // of the sequence's first row
    int32_t key, key_end;       // keys: from a multiple of 32 on
    uint32_t part, parts;       // this workgroup's part of the keys, parts that are not empty
};

// part: which of p.parts.  LAST_FIRST: a sequence's tiles from the last, which sees most, to the first.
template <bool LAST_FIRST>
__device__ inline bool find_columns(const AttentionProblem &p, uint32_t t, uint32_t part, ColumnTile &c)
{
    const uint32_t G = p.seq.Hq / p.seq.Hkv;
    c.part = part;
    c.head = t % p.seq.Hkv;
    SequenceTile at;
    if (!find_sequence(p.seq, t / p.seq.Hkv, ColumnBase{G, p.columns}, p.max_len, at)) return false;
    c.s = at.s;
    c.row = at.row;
    c.n = at.n;
    const uint32_t tiles = (c.n * G + p.columns - 1) / p.columns;
    if (at.tile >= tiles) return false;
    c.first = (LAST_FIRST ? tiles - 1 - at.tile : at.tile) * p.columns;
    c.end = min(c.first + p.columns, c.n * G);
    c.position = at.length - (int32_t)c.n;
    c.key_end = max(c.position + (int32_t)((c.end - 1) / G) + 1, 0);
    c.key = p.window ? max(c.position + (int32_t)(c.first / G) - window_of(p) + 1, 0) & ~31 : 0;
    c.parts = c.key_end > c.key ? ((uint32_t)(c.key_end - c.key) + p.part - 1) / p.part : 0;
    return true;
}

// The keys that a column sees: those after `low`, up to `high`.
struct Sight {
    int32_t low, high;
    __device__ bool sees(int32_t key) const { return key > low && key <= high; }
};
__device__ inline Sight sight_of(const AttentionProblem &p, int32_t position) { return {p.window ? position - window_of(p) : -1, position}; }

// Weights of one largest score relative to another; 0 where nothing was seen.
__device__ inline float rescale(float from, float to) { return __builtin_amdgcn_exp2f(from - (to == -INFINITY ? 0.0f : to)); }

__device__ inline bf16x8 as_fragment(u32x4 w) { return __builtin_bit_cast(bf16x8, w); }

// An infinity or a NaN among eight bf16?
__device__ inline bool any_special(u32x4 w)
{
    bool special = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) special |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return special;
}

// Eight tokens of which the first `count` are meant: zeros in place of the others.
__device__ inline u32x4 first_tokens(u32x4 w, int32_t count)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = count >= 2 * i + 2 ? w[i] : count == 2 * i + 1 ? w[i] & 0xffffu : 0u;
    return w;
}

}  // namespace salus
