// The 4-bit cache of keys and values: its grid, the words that hold it and where a token's row lies.  Shared by the kernels that
// write it, read it and attend over it.
#pragma once
#include "lowbit.h"

namespace fobq {

// A grid word: the scale, a positive bf16, in the high half (the word with its low half cleared is the scale as fp32), the zero
// point 0 .. 15 in the lowest four bits.
__host__ __device__ inline uint32_t kv4_zero(uint32_t word) { return word & 15u; }

// The page that holds token t of a sequence, or -1: behind the table, or an entry that is no page of the cache.  No kernel forms an
// address from an entry that did not pass here.
__host__ __device__ inline int kv4_page(const int32_t* row, int max_pages, int pages, int shift, int t)
{
    const unsigned at = (unsigned)t >> shift;       // (a negative t is far behind any table)
    if (at >= (unsigned)max_pages) return -1;
    const int page = row[at];
    return (unsigned)page < (unsigned)pages ? page : -1;
}

// Sequence b of packed rows has rows [first, first + count): starts as the caller gave them, kept inside 0 .. rows.
struct Kv4Rows { int first, count; };
__host__ __device__ inline Kv4Rows kv4_rows(const int32_t* starts, int b, int rows)
{
    if (!starts) return b < rows ? Kv4Rows{b, 1} : Kv4Rows{rows, 0};
    int lo = starts[b], hi = starts[b + 1];
    lo = lo < 0 ? 0 : (lo > rows ? rows : lo);
    hi = hi < lo ? lo : (hi > rows ? rows : hi);
    return Kv4Rows{lo, hi - lo};
}

// Tokens of sequence b, as the caller says (its new rows are the last of them), and the most that its table has places for: those behind
// are not there.
__host__ __device__ inline int kv4_length(const int32_t* lengths, int b) { return lengths[b] < 0 ? 0 : lengths[b]; }
__host__ __device__ inline int kv4_places(int max_pages, int shift) { return max_pages << shift; }       // below 2^30

// Where packed row `row` of sequence b lies: its page (-1: none) and its place there.
struct Kv4Place { int page, place; };
__host__ __device__ inline Kv4Place kv4_place(const Kv4Seqs& s, int pages, int shift, int b, int row)
{
    const Kv4Rows r = kv4_rows(s.starts, b, s.rows);
    if (row < r.first || row >= r.first + r.count) return Kv4Place{-1, 0};
    const int t = kv4_length(s.lengths, b) - r.count + (row - r.first);
    if (t < 0) return Kv4Place{-1, 0};
    return Kv4Place{kv4_page(s.table + (int64_t)b * s.table_ld, s.max_pages, pages, shift, t), t & ((1 << shift) - 1)};
}

#ifdef __HIPCC__
// The largest b in [0, n) with at(b) <= x for an at() that does not decrease (0 if there is none): all 64 lanes of a wavefront look at
// once, so that up to 64 sequences take one round trip to memory and 4096 two (one lane alone: six and twelve).
template <class F>
__device__ __forceinline__ int wave_search(int n, int64_t x, F at)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int b = lo + (lane + 1) * step;
        const int k = __popcll(__ballot(b < hi && at(b) <= x));
        lo += k * step;
        hi = hi < lo + step ? hi : lo + step;
    }
    return lo;
}
#endif

}  // namespace fobq
