// A paged key/value cache in 4 bits: where a token's codes lie, which tokens a call is about, and how attention cuts its work.  Host and
// device arithmetic; what a caller's arrays on the device say (page_table, lengths, begins) is checked here before it becomes an address.
#pragma once
#include <stdint.h>

#include "hq.h"

namespace hq {

__host__ __device__ __forceinline__ int kv4_pitch(int d) { return (d + 31) & ~31; }
__host__ __device__ __forceinline__ int kv4_min(int a, int b) { return a < b ? a : b; }
__host__ __device__ __forceinline__ int kv4_max(int a, int b) { return a > b ? a : b; }

struct Kv4 {
    uint8_t *k, *v;             // [pages, kv_heads, page_size, pitch / 2], [pages, kv_heads, page_size / 8, pitch, 4]
    float *k_scale, *v_scale;   // [pages, kv_heads, page_size]
    const int32_t *table, *lengths, *begins;
    int64_t pages;
    int page_log2, kv_heads, d, pitch, block_log2, batch, table_pages, t, each;   // each: tokens of a sequence where begins is null

    // The first token of sequence s; of `batch`: the end of the last.  In 0 .. t whatever begins holds.
    __host__ __device__ __forceinline__ int begin(int s) const {
        if (s == 0) return 0;
        if (!begins) return s * each;
        return kv4_max(0, kv4_min(begins[s], t));
    }
    __host__ __device__ __forceinline__ int capacity() const { return table_pages << page_log2; }   // (tokens; the host checks that it fits)
    // The page of a position; -1 for a position without one.  entry: reads an entry of the sequence's table.
    template <class F> __host__ __device__ __forceinline__ int64_t checked(int position, F entry) const {
        if (position < 0 || position >= capacity()) return -1;
        const int64_t p = entry(position >> page_log2);
        return p < pages ? (p < 0 ? -1 : p) : -1;
    }
    __host__ __device__ __forceinline__ int64_t page(int s, int position) const {
        return checked(position, [&](int column) { return table[static_cast<int64_t>(s) * table_pages + column]; });
    }
    // The first slot of a head of a page: slots are tokens (scales), pitch / 2 bytes of k, a group of 8 of them 4 pitch bytes of v.
    __host__ __device__ __forceinline__ int64_t slots(int64_t page, int head) const { return (page * kv_heads + head) << page_log2; }
    __host__ __device__ __forceinline__ int slot(int position) const { return position & ((1 << page_log2) - 1); }
    __host__ __device__ __forceinline__ int64_t row_bytes() const { return pitch >> 1; }
};

// Positions are worked on in aligned groups of 8 (a channel's codes of a group share a dword of v), a workgroup each.  Sequence s has the
// groups from group_begin(s) on, at least as many as its tokens touch; behind the last sequence come groups of tokens of none.
__host__ __device__ __forceinline__ int kv4_group_begin(int first_token, int s) { return (first_token >> 3) + 2 * s; }
__host__ __device__ __forceinline__ int kv4_groups(int t, int batch) { return (t >> 3) + 2 * batch + 2; }

// The tokens of a group: `count` rows from token `row` on, at positions from `position` on, which are all in one group of 8.
struct Kv4Group {
    int s;           // sequence; batch: none
    int row, count;
    int position;    // (of tokens of no sequence: meaningless)
};
// The sequence that group `index` belongs to where begins is null: the last s with s each / 8 + 2 s <= index, at most `batch`.
__host__ __device__ __forceinline__ int kv4_sequence(const Kv4 &c, int index) {
    // s (each / 8 + 2) is between the left side and one less, so the quotient is s or one too small
    int s = kv4_min(static_cast<int>(static_cast<uint32_t>(index) * 8u / static_cast<uint32_t>(c.each + 16)), c.batch);
    while (s < c.batch && kv4_group_begin(c.begin(s + 1), s + 1) <= index) ++s;
    return s;
}
// begin, end: of sequence s; read: reads a number of lengths.
template <class F>
__host__ __device__ __forceinline__ Kv4Group kv4_group(const Kv4 &c, int s, int begin, int end, int index, F read) {
    const int j = index - kv4_group_begin(begin, s);
    if (s >= c.batch) {
        const int64_t row = begin + int64_t{8} * j;
        return row < c.t ? Kv4Group{s, static_cast<int>(row), kv4_min(8, c.t - static_cast<int>(row)), 0} : Kv4Group{s, 0, 0, 0};
    }
    const int n = end - begin, length = kv4_max(0, read(c.lengths + s));
    const int64_t first = int64_t{length} - n;                       // position of the sequence's first token; negative: no place for it
    const int64_t group = ((first >> 3) + j) * 8;
    const int64_t from = group > first ? group : first, to = group + 8 < length ? group + 8 : length;
    if (n <= 0 || j < 0 || from >= to) return {s, 0, 0, 0};
    return {s, begin + static_cast<int>(from - first), static_cast<int>(to - from), static_cast<int>(from)};
}

// The positions that a query at `position` sees: those below `sinks`, and from `from` to itself.
struct Kv4Seen {
    int sinks, from;
};
__host__ __device__ __forceinline__ Kv4Seen kv4_seen(int position, int window, int sinks) {
    const int from = window > 0 && position >= window ? position - window + 1 : 0;
    return {kv4_min(sinks, from), from};
}

// Attention's rows: row r of a sequence and key head is its new token r / group under query head r % group of that key head; a workgroup
// takes rows() of them over a part of their tokens, in steps of 32 tokens for a wave.  Parts are cut so that about `target` workgroups share
// the steps of all rows, none much shorter than `least` steps.
struct Kv4Cut {
    int rows_log2, waves_log2, group, target, least, window, sinks;
    int reach;                                                  // tokens that a block of rows sees at most; window and sinks with ragged ends
    uint32_t magic, shift;                                      // exact division by group
    __host__ __device__ __forceinline__ int token_of(int row) const {
        return group == 1 ? row : static_cast<int>(static_cast<uint32_t>(uint64_t{static_cast<uint32_t>(row)} * magic >> 32) >> shift);
    }
    __host__ __device__ __forceinline__ int rows() const { return 1 << rows_log2; }
};
inline int kv4_reach(int window, int sinks, int rows, int group) {
    const int64_t most = int64_t{window} + sinks + (rows + group - 1) / group + 64;   // (64: the ragged ends of both ranges)
    return window > 0 && most < 0x7FFFFFFF ? static_cast<int>(most) : 0x7FFFFFFF;
}
struct Kv4Span {        // of a sequence: blocks of rows, and the steps through the tokens that the largest of them looks at
    int begin, n, length, blocks, steps;
};
__host__ __device__ __forceinline__ Kv4Span kv4_span(const Kv4 &c, const Kv4Cut &cut, int s) {
    const int length = kv4_max(0, c.lengths[s]), begin = c.begin(s), n = kv4_max(0, c.begin(s + 1) - begin);
    const int blocks = static_cast<int>((static_cast<uint32_t>(n) * cut.group + cut.rows() - 1) >> cut.rows_log2);   // (t x heads is below 2^31)
    const int tokens = kv4_min(kv4_min(length, c.capacity()), cut.reach);
    // rows for one wave are given to all waves, which share the tokens
    const bool apart = static_cast<uint32_t>(n) * cut.group <= static_cast<uint32_t>(cut.rows() >> cut.waves_log2);
    return {begin, n, length, blocks, static_cast<int>((static_cast<uint32_t>(tokens) + 31) >> (apart ? 5 + cut.waves_log2 : 5))};
}
constexpr int kKv4Undivided = 0x7FFFFFFF;   // no sequence has more steps than a part
// work: steps times blocks of rows of all sequences, for one key head, by a sum of up to 2^18 floats: the share is enlarged by more than that
// sum can be too small
__host__ __device__ __forceinline__ int kv4_part(const Kv4Cut &cut, float work, int kv_heads) {
    const float share = work * static_cast<float>(kv_heads) / static_cast<float>(cut.target) * 1.03125f + 1.0f;
    if (!(share < 0x1p30f)) return kKv4Undivided;
    return kv4_max(static_cast<int>(share), cut.least);
}
// (to the nearest: no part of less than two thirds)
__host__ __device__ __forceinline__ int kv4_parts(const Kv4Span &p, int part) {
    const uint32_t parts = (static_cast<uint32_t>(p.steps) + (static_cast<uint32_t>(part) >> 1)) / static_cast<uint32_t>(part);
    return parts > 1 ? static_cast<int>(parts) : 1;
}

// The tokens that a block of rows looks at, in tiles of 32 positions: those of the sinks (tiles 0 .. sinks - 1) and those from `from` to `to`.
struct Kv4Tiles {
    int sinks, from, to;
    __host__ __device__ __forceinline__ int count() const { return sinks + (to - from); }
    __host__ __device__ __forceinline__ int tile(int i) const { return i < sinks ? i : from + (i - sinks); }
};
// first, last: positions of the block's first and last row (the last may be negative: nothing is seen)
__host__ __device__ __forceinline__ Kv4Tiles kv4_tiles(int first, int last, int window, int sinks) {
    if (last < 0) return {0, 0, 0};
    const int to = (last >> 5) + 1;
    const Kv4Seen s = kv4_seen(kv4_max(first, 0), window, sinks);
    const int from = s.from >> 5;
    // (a later row of the block can see sinks that the first one has in its window: tiles before `from` are enough)
    const int before = kv4_min((kv4_seen(last, window, sinks).sinks + 31) >> 5, from);
    return {before, from, to};
}

}  // namespace hq
