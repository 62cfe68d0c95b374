// Attention of packed query rows over the 4-bit cache: out = softmax(scale q K^T + mask) V, K and V = scale_t (code - zero_t) per token.
//
// One pass over the tokens with the running maximum and sum of the softmax, 32 tokens at a time, everything in registers:
//   S^T = K Q^T   16x16x32 matrix instructions, tokens x query rows.  K enters as codes: S = scale_k (sum q code' - zero' sum q),
//                 code' and zero' with the offset of the trick below, sum q taken once.  Only the query rows are rounded
//                 numbers here, the sums are in fp32.
//   O^T += V^T P^T  channels x query rows.  P = exp2(S - m) scale_v in fp16 (11 bits), V as code - zero, exact in fp16.
// Codes become 16-bit floats without conversions: four bits under the exponent of 128 (bf16, 7 bits of mantissa) or 1024 (fp16) are
// 128 + code; fp16 also takes the upper four bits of a byte (1024 + 16 code), so every other code needs no shift.
//
// The order of a contraction is free as long as both sides keep it.  A lane (column c = lane % 16, quarter g = lane / 16) holds after
// S^T the tokens 8 g .. 8 g + 7 of one query row; those are the eight it multiplies next, so P never leaves its lane, and the rows of
// K are dealt to the instruction's rows accordingly.  V's row n is the n-th piece of dim / 16 channels of a token, read as that, and
// the lane transposes 8 tokens x dim / 16 codes by byte selects.  A lane's results are dim / 4 consecutive channels of one query row.
//
// fp16 weights and the range of V: m follows the running maximum of S + log2 scale_v (its whole part), not of S, so that a row's largest
// weights are near 1 whatever the size of the values, and enter fp16 2^6 up, where the largest still fit (below 2^15) and those down to 2^-20 of
// it keep all 11 bits, the others down to 2^-31 some: a long tail behind a few strong tokens is made of such.  The sum of the softmax has the same m, raised by 2^28 (scale_v takes that off P again):
// with scales up to 2^127 its largest terms are still 2^27 times what fp32 can hold, with scales down to 2^-60 2^31 of them are finite.
// Smaller scales count as 2^-60 in m, so that values below 2^-80 lose bits.
// The maximum is raised only when it is exceeded by 2^8: most tiles of 32 tokens then rescale nothing.
#include "kv4.h"

#include <algorithm>
#include <type_traits>

namespace fobq {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

constexpr float NEG_MAX = -3.402823466e38f;
constexpr int VALUE_FLOOR = -60;
constexpr float BIAS = 28.f, BIAS2 = 268435456.f;       // and 2^BIAS
constexpr float LIFT = 64.f;            // what fp16 weights are taken up by: the largest is below 2 * 2^RAISE * LIFT = 2^15
constexpr float RAISE = 8.f;            // binary orders of magnitude that a score may exceed the running maximum by
constexpr int KV4_PART = 256;           // tokens of a part at least: eight tiles, two for each wavefront that shares the rows
// Sequences of no more tokens than these are not split: one launch, not two, and no scratch.  (8 of 600 tokens, from call to call: 11 us,
// 16 split; 32 of 1024: 16, 18.  At 2048 it turns: 16 sequences 19.5 us, 18.3 split; 8 with 8 new tokens each 24, 18.)
constexpr int KV4_UNSPLIT = 1024;
constexpr int KV4_MAX_PARTS = 64;       // a lane each where they are joined
constexpr int KV4_SPLIT_SEQS = 256;     // more sequences than these are not split: they fill the chip
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;

struct AttnArgs {
    Kv4View c; Kv4Seqs s; Kv4Query q;
    int heads_q, tile;     // query heads; query rows of a workgroup
    int slots;             // workgroups of a head where sequences are split (0: none is)
    float scale2;          // scale * log2(e)
    float* part_o;         // heads x slots x tile x dim: sums of the rows of a split sequence's part
    float* part_ml;        // the same without dim: maximum (in binary orders) and sum of the weights
    int2* seqs;            // per sequence its first workgroup and its parts, for the launch that joins them
};

// How the sequences are split into parts of about equal size, which the host cannot know: the lengths are on the device.  A sequence has
// one workgroup per tile of its rows and part of its tokens, up to KV4_MAX_PARTS parts of KV4_PART tokens at least; the longest part is
// about as short as it can be with all of them in the slots that there are, which the chip holds at a time (six halvings: to 1 / 64 of the
// distance between a length that is too short and one that fits for sure).  Every wavefront works this out for itself, a lane to a sequence.  (32 sequences of 5000 to
// 16000 tokens in as many parts each take 88 us, so 82; 8 of 16384 in three times as many parts 48, so 40.)
struct Split {
    static constexpr int J = KV4_SPLIT_SEQS / 64;
    int row[J], count[J], length[J], parts[J], first[J], items[J];   // of sequence 64 j + lane: its packed rows, its tokens, its parts; its
                                                                     // slots are first .. first + items - 1
};
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_dpp(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
// the sum over the lanes up to this one
__device__ __forceinline__ int sum_to_lane(int x)
{
    x = add_dpp<0x111, 0xf>(x);              // the lane below in a row of 16, two, four, eight below
    x = add_dpp<0x112, 0xf>(x);
    x = add_dpp<0x114, 0xf>(x);
    x = add_dpp<0x118, 0xf>(x);
    x = add_dpp<0x142, 0xa>(x);              // the last lane of the row below, to the second and fourth row
    return add_dpp<0x143, 0xc>(x);           // of the second row, to the upper half
}
__device__ __forceinline__ Split split_of(const AttnArgs& a)
{
    constexpr int J = Split::J;
    const int lane = threadIdx.x & 63;
    Split s;
    int tiles[J], spans[J], low = 0, high = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int b = 64 * j + lane;
        s.row[j] = s.count[j] = s.length[j] = tiles[j] = spans[j] = 0;
        if (64 * j < a.s.n_seqs && b < a.s.n_seqs) {
            const Kv4Rows r = kv4_rows(a.s.starts, b, a.s.rows);
            s.row[j] = r.first;
            s.count[j] = r.count;
            s.length[j] = kv4_length(a.s.lengths, b);
            const int held = min(s.length[j], kv4_places(a.s.max_pages, a.c.shift));
            const int tokens = a.q.window > 0 ? (int)min((int64_t)held, (int64_t)a.q.window + r.count) : held;
            tiles[j] = (r.count * a.q.group + a.tile - 1) / a.tile;
            spans[j] = (tokens + 31) / 32;
            // (starts out of order could make more tiles than there are slots: those are cut off, here and where they are joined)
            const uint64_t work = (uint64_t)min(tiles[j], a.slots) * spans[j];       // below 2^17 * 2^25
            low += (int)(work & 0xffff);
            high += (int)(work >> 16);
        }
    }
    low = __builtin_amdgcn_readlane(sum_to_lane(low), 63);
    high = __builtin_amdgcn_readlane(sum_to_lane(high), 63);
    const float total = (float)high * 65536.f + (float)low;
    // parts of sequence 64 j + lane if none is longer than `span` tiles of 32 tokens
    auto parts_at = [&](int j, int span) { return max(1, min(KV4_MAX_PARTS, (int)((unsigned)(spans[j] + span - 1) / (unsigned)span))); };
    auto fits = [&](int span) {
        int sum = 0;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (64 * j < a.s.n_seqs) sum += min(tiles[j], a.slots) * parts_at(j, span);
        return __builtin_amdgcn_readlane(sum_to_lane(sum), 63) <= a.slots;
    };
    int all = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) all += min(tiles[j], a.slots);
    const int spare = a.slots - __builtin_amdgcn_readlane(sum_to_lane(all), 63);
    // between the whole work over all slots, and over those that are left when every tile has one (which always fits)
    int span = spare > 0 ? (int)fminf(total / (float)spare * 1.000001f + 2.f, 1e9f) : 1 << 30, below = (int)(total / (float)a.slots) - 1;
    span = max(span, KV4_PART / 32);
    below = max(below, KV4_PART / 32 - 1);
    for (int i = 0; i < 6 && below + 1 < span; ++i) {
        const int mid = below + (span - below) / 2;
        if (fits(mid)) span = mid;
        else below = mid;
    }
    int before = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        s.parts[j] = 1;
        s.items[j] = s.first[j] = 0;
        if (64 * j >= a.s.n_seqs) continue;
        s.parts[j] = parts_at(j, span);
        s.items[j] = min(tiles[j], a.slots) * s.parts[j];
        const int sum = sum_to_lane(s.items[j]);
        s.first[j] = before + sum - s.items[j];
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return s;
}

// (x & mask) | bits is one instruction where the compiler has the mask in a scalar register and the bits in a vector one; as two
// literals they cost an instruction each.  So the bits are made where it cannot see what they are.  (The instruction itself is left to the
// compiler: between it and a matrix instruction that reads its result there have to be wait states, which inline asm does not get.)
struct Bits { uint32_t b128, h1024, h64; };
__device__ __forceinline__ Bits offset_bits()
{
    Bits b{0x43004300u, 0x64006400u, 0x54005400u};
    asm("" : "+v"(b.b128), "+v"(b.h1024), "+v"(b.h64));
    return b;
}
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) { return (x & mask) | bits; }
constexpr uint32_t LOW = 0x000f000fu, HIGH = 0x00f000f0u;

template <class T> struct Frag;
template <> struct Frag<bf16_t> {
    static __device__ __forceinline__ f4 mfma(u4 a, u4 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static constexpr float OFFSET = 128.f;
    // 8 codes as 128 + code: register j has codes j and j + 4
    static __device__ __forceinline__ u4 codes(uint32_t w, const Bits& b)
    {
        u4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = and_or(w >> (4 * j), LOW, b.b128);
        return r;
    }
};
template <> struct Frag<f16_t> {
    static __device__ __forceinline__ f4 mfma(u4 a, u4 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static constexpr float OFFSET = 0.f;
    // 8 codes as they are
    static __device__ __forceinline__ u4 codes(uint32_t w, const Bits& b)
    {
        u4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = j < 2 ? w : w >> 8;
            const h2 v = j & 1 ? __builtin_elementwise_fma(__builtin_bit_cast(h2, and_or(x, HIGH, b.h1024)), h2{(f16_t)0.0625f, (f16_t)0.0625f},
                                                           h2{(f16_t)-64.f, (f16_t)-64.f})
                               : __builtin_bit_cast(h2, and_or(x, LOW, b.h1024)) + h2{(f16_t)-1024.f, (f16_t)-1024.f};
            r[j] = __builtin_bit_cast(uint32_t, v);
        }
        return r;
    }
};

// over the four lanes of a column, a quarter of the wavefront apart: the swaps put the other half, then the other quarter, beside each lane's own
template <class F>
__device__ __forceinline__ float quarters(float x, F f)
{
    uint32_t u = __float_as_uint(x);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    u = __float_as_uint(f(__uint_as_float(r[0]), __uint_as_float(r[1])));
    r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quarters_max(float x) { return quarters(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float quarters_sum(float x) { return quarters(x, [](float a, float b) { return a + b; }); }

// lane E of every quarter, to the whole quarter (as an operand of the instruction that uses it)
template <int E>
__device__ __forceinline__ float from_lane(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x150 + E, 0xf, 0xf, true));
}
template <int E = 0, class F>
__device__ __forceinline__ void for8(F f)
{
    if constexpr (E < 8) {
        f(std::integral_constant<int, E>());
        for8<E + 1>(f);
    }
}

// The pages of 32 tokens: of the first and the last 16 of them, as pages have 16 tokens at least.
struct Pages { int first, last; };
// A sequence's row of the table, 64 entries in the lanes of a wavefront (-1: no page): a page is a read of a lane, and memory is asked once
// in 64 pages.
struct PageRow {
    const int32_t* __restrict__ row;
    int have = -1, entries = -1;           // which 64 of them; (per lane) the entry
    __device__ __forceinline__ int page(const Kv4View& c, int max_pages, int t)
    {
        const int at = __builtin_amdgcn_readfirstlane(t >> c.shift);
        if (at >> 6 != have) {
            have = at >> 6;
            entries = kv4_page(row, max_pages, c.pages, 0, 64 * have + (threadIdx.x & 63));
        }
        return __builtin_amdgcn_readlane(entries, at & 63);
    }
    __device__ __forceinline__ Pages pages(const Kv4View& c, int max_pages, int t0)
    {
        const int first = page(c, max_pages, t0);
        return Pages{first, c.shift > 4 ? first : page(c, max_pages, t0 + 16)};
    }
};

// 32 tokens of one head: where their rows are, and the grids of token 8 g + lane % 8.
struct Where {
    int64_t row0, row1;        // the cache rows of token 0, and (pages of 16) of token 16, less 16
    bool first, last;          // whether the first and the last 16 tokens lie on a page
};
__device__ __forceinline__ Where where(const Kv4View& c, Pages p, int h, int t0)
{
    // tokens on no page: page 0 is read in their place, and masked
    const int mask = (1 << c.shift) - 1;
    Where w;
    w.first = p.first >= 0;
    w.last = p.last >= 0;
    w.row0 = ((((int64_t)(w.first ? p.first : 0)) * c.heads + h) << c.shift) + (t0 & mask);
    w.row1 = c.shift > 4 ? w.row0 : ((((int64_t)(w.last ? p.last : 0)) * c.heads + h) << c.shift) + ((t0 + 16) & mask) - 16;
    return w;
}
// f(row of token 0), for a lane whose tokens are among the first or the last 16.  With pages of 32 tokens or more the row is a scalar.
template <class F>
__device__ __forceinline__ void at_token(const Kv4View& c, const Where& w, bool second, F f)
{
    const int64_t row0 = w.row0, row1 = w.row1;
    if (c.shift > 4) f(row0);
    else f(second ? row1 : row0);
}

struct Grids {
    uint32_t k, v;             // of token 8 g + lane % 8
    bool first, last;          // whether the first and the last 16 tokens lie on a page
};

template <int D> struct Tokens {
    static constexpr int K = D / 32, V = D / 128 > 0 ? D / 128 : 1;   // words of a K row, words of a V row (dim 64: half a word)
    uint32_t k[2][K];
    uint32_t v[8][V];
    Grids grids;
};

__device__ __forceinline__ void load_grids(const Kv4View& c, const Where& w, Grids& x)
{
    x.first = w.first;
    x.last = w.last;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const unsigned at = 8 * g + (lane & 7);
    at_token(c, w, g & 2, [&](int64_t row) {
        x.k = (c.k_grids + row)[at];
        x.v = (c.v_grids + row)[at];
    });
}

template <int D>
__device__ __forceinline__ void load_tokens(const Kv4View& c, Pages p, int h, int t0, Tokens<D>& x)
{
    constexpr int ROW = D / 2;
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const Where w = where(c, p, h, t0);
    // K: row r of instruction i is token 8 (r / 4) + 4 i + r % 4; V: row e of quarter g is token 8 g + e
    at_token(c, w, r & 8, [&](int64_t row) {
        const uint8_t* __restrict__ k = c.k_codes + row * ROW;
        const unsigned off = (8 * (r >> 2) + (r & 3)) * ROW + 4 * Tokens<D>::K * g;
#pragma unroll
        for (int i = 0; i < 2; ++i) __builtin_memcpy(x.k[i], __builtin_assume_aligned(k + off + 4 * i * ROW, D == 64 ? 8 : 16), sizeof x.k[i]);
    });
    at_token(c, w, g & 2, [&](int64_t row) {
        const uint8_t* __restrict__ v = c.v_codes + row * ROW;
        const unsigned off = 8 * g * ROW + (D / 32) * r;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (D == 64) x.v[e][0] = *reinterpret_cast<const uint16_t*>(v + off + e * ROW);
            else __builtin_memcpy(x.v[e], __builtin_assume_aligned(v + off + e * ROW, 4 * Tokens<D>::V), sizeof x.v[e]);
        }
    });
    load_grids(c, w, x.grids);
}

// The index-th tile of rows, those that see most tokens first (causal; the workgroups that start last then have least to do): its
// sequence (-1: there are not so many) and its number there.  A tile's level is how many tiles of tokens the sequence has up to its own; the
// levels are searched for the one that the index falls into.  (3 prompts of 2048 tokens take
// 12 % less time than in the order of the sequences, 6 of up to 1000 behind 2000 9 %.)
struct Ranked { int b, tile; Kv4Rows rows; int length; };
__device__ __forceinline__ Ranked ranked(const AttnArgs& a, int tile_rows, int index)
{
    constexpr int J = KV4_SPLIT_SEQS / 64;
    const int lane = threadIdx.x & 63;
    int row[J], count[J], length[J], tiles[J], base[J], top = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int b = 64 * j + lane;
        row[j] = count[j] = length[j] = tiles[j] = base[j] = 0;
        if (64 * j < a.s.n_seqs && b < a.s.n_seqs) {
            const Kv4Rows r = kv4_rows(a.s.starts, b, a.s.rows);
            row[j] = r.first;
            count[j] = r.count;
            length[j] = kv4_length(a.s.lengths, b);
            tiles[j] = (int)(((int64_t)r.count * a.q.group + tile_rows - 1) / tile_rows);
            base[j] = (int)min((int64_t)max(0, length[j] - r.count) * a.q.group / tile_rows, (int64_t)(1 << 30) - 1);
            top = max(top, base[j] + tiles[j]);
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, __shfl_xor(top, off));
    // tiles at `level` and above
    auto above = [&](int level) {
        int sum = 0;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (64 * j < a.s.n_seqs) sum += min(tiles[j], max(0, base[j] + tiles[j] - level));
        return __builtin_amdgcn_readlane(sum_to_lane(sum), 63);
    };
    int level = 0, over = __builtin_amdgcn_readfirstlane(top), higher = 0;
    Ranked x{-1, 0, Kv4Rows{0, 0}, 0};
    if (above(0) <= index) return x;
    while (over - level > 1) {
        const int mid = level + (over - level) / 2, n = above(mid);
        if (n > index) level = mid;
        else { over = mid; higher = n; }
    }
    int left = index - higher;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const bool in = base[j] <= level && level < base[j] + tiles[j];
        const uint64_t all = __ballot(in);
        const int place = __builtin_amdgcn_mbcnt_hi((unsigned)(all >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)all, 0));
        const uint64_t hit = __ballot(in && place == left);
        if (hit) {
            const int at = __ffsll((unsigned long long)hit) - 1;
            x.b = 64 * j + at;
            x.tile = level - __builtin_amdgcn_readlane(base[j], at);
            x.rows = Kv4Rows{__builtin_amdgcn_readlane(row[j], at), __builtin_amdgcn_readlane(count[j], at)};
            x.length = __builtin_amdgcn_readlane(length[j], at);
        }
        left -= __popcll(all);
    }
    return x;
}

// What is taken off the values' codes, as fp16 with their offset: 1024 + zero for codes in the low half of a byte, 64 + zero (of
// (1024 + 16 code) / 16) in the high half; of tokens 2 j and 2 j + 1 of the lane's eight.
struct Zeros { h2 low[4], high[4]; };
__device__ __forceinline__ Zeros value_zeros(uint32_t vg, const Bits& b)
{
    // a lane's own zero and its neighbour's (tokens 2 j and 2 j + 1 in lanes 2 j), then lane 2 j's to everybody
    const uint32_t next = __builtin_amdgcn_mov_dpp(vg, 0xB1, 0xf, 0xf, true), both = __builtin_amdgcn_perm(next, vg, 0x05040100u);
    const float low = __uint_as_float(and_or(both, LOW, b.h1024)), high = __uint_as_float(and_or(both << 4, HIGH, b.h64));
    Zeros z;
    for8([&](auto e) {
        constexpr int E = decltype(e)::value;
        if constexpr (E % 2 == 0) {
            z.low[E / 2] = __builtin_bit_cast(h2, from_lane<E>(low));
            z.high[E / 2] = __builtin_bit_cast(h2, from_lane<E>(high));
        }
    });
    return z;
}
// code - zero of channel n (of four) of the lane's eight tokens; pair[j]: the four channels' codes of tokens 2 j and 2 j + 1
__device__ __forceinline__ u4 value_fragment(const uint32_t (&pair)[4], int n, const Zeros& z, const Bits& b)
{
    u4 vf;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = n < 2 ? pair[j] : pair[j] >> 8;
        const h2 v = n & 1 ? __builtin_elementwise_fma(__builtin_bit_cast(h2, and_or(w, HIGH, b.h1024)), h2{(f16_t)0.0625f, (f16_t)0.0625f}, -z.high[j])
                           : __builtin_bit_cast(h2, and_or(w, LOW, b.h1024)) - z.low[j];
        vf[j] = __builtin_bit_cast(uint32_t, v);
    }
    return vf;
}

// WAVES wavefronts, each with QT x 16 query rows.
//   SHARE: the same rows for all of them; each takes every WAVES-th tile of tokens into its registers, and their sums meet in LDS at the
//     end.  For few rows, where the tokens are what costs.  (32 sequences of up to 16384 tokens, 8 heads of 128, 4 query heads each: 75 us, 4.7 TB/s
//     of codes and grids, where a large copy has 4.9; 16384 each 117 us, 4.9 TB/s.)
//   otherwise: rows of its own.  All need the same tokens: each turns a quarter of a stage's codes into fragments in LDS, a stage ahead,
//     and reads all of them.  A stage is 64 tokens (dim 256: 32, for 64 KiB of LDS), with a barrier each: a wavefront's loads are then 16 bytes of
//     K and whole pairs of bytes of V, and turning them takes 40 vector instructions for 32 tokens, the softmax of 32 rows 160.  These
//     bound it: of 2.46 GHz, the vector units issue for 61 % and the matrix units work for 29 % of the time, with two wavefronts a
//     SIMD (3 prompts of about 2048 tokens behind as many, 32 query heads: 347 us, 745 TFLOP/s; with 32 tokens a stage 389; with eight
//     wavefronts a workgroup, which turn half as many codes each but keep in step, 406).
template <class T, int D, int QT, bool SHARE>
__global__ __launch_bounds__(256, 2) void kv4_attention_kernel(AttnArgs a)
{
    constexpr int WAVES = 4, M = D / 16, TILE = 16 * QT * (SHARE ? 1 : WAVES);
    __shared__ __attribute__((aligned(16))) float sh_o[SHARE ? WAVES : 1][SHARE ? 16 * QT * (D + 4) : 4];
    __shared__ float sh_ml[SHARE ? WAVES : 1][SHARE ? 16 * QT * 2 : 1];
    constexpr int SUB = D == 256 ? 1 : 2;
    __shared__ u4 sh_f[SHARE ? 1 : 2][SHARE ? 1 : SUB * 2 * M][SHARE ? 1 : 64];   // per tile of 32 tokens the fragments of K, then of V

    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = a.q.group;
    const Bits bits = offset_bits();

    // the sequence, the tile of its rows and the part of its tokens that this workgroup has
    const int h = blockIdx.x % a.c.heads, index = blockIdx.x / a.c.heads;
    int b = -1, part = 0, parts = 1, tile_of_rows = 0, length = 0;
    Kv4Rows mine{0, 0};
    if (a.slots) {
        const Split split = split_of(a);
#pragma unroll
        for (int j = 0; j < Split::J; ++j)
            if (blockIdx.x == 0 && wave == 0 && 64 * j + lane < a.s.n_seqs) a.seqs[64 * j + lane] = int2{split.first[j], split.parts[j]};
#pragma unroll
        for (int j = 0; j < Split::J; ++j) {
            const uint64_t hit = __ballot(index >= split.first[j] && index < split.first[j] + split.items[j]);
            if (hit) {
                const int at = __ffsll((unsigned long long)hit) - 1;
                b = 64 * j + at;
                mine = Kv4Rows{__builtin_amdgcn_readlane(split.row[j], at), __builtin_amdgcn_readlane(split.count[j], at)};
                length = __builtin_amdgcn_readlane(split.length[j], at);
                parts = __builtin_amdgcn_readlane(split.parts[j], at);
                const int i = index - __builtin_amdgcn_readlane(split.first[j], at);
                tile_of_rows = i / parts;
                part = i - tile_of_rows * parts;
            }
        }
        if (b < 0) return;
    } else if (!SHARE && a.s.n_seqs <= KV4_SPLIT_SEQS) {
        const Ranked x = ranked(a, TILE, index);
        b = x.b;
        mine = x.rows;
        length = x.length;
        tile_of_rows = x.tile;
        if (b < 0) return;
    } else {
        // sequence b's tiles begin at floor(first row * G / TILE) + b, which leaves room for every sequence's last, partial tile; with
        // many rows the last tiles first, which see most
        auto first_tile = [&](int i) { return (int64_t)kv4_rows(a.s.starts, i, a.s.rows).first * G / TILE + i; };
        const int place = SHARE ? index : (int)(gridDim.x / a.c.heads) - 1 - index;
        b = __builtin_amdgcn_readfirstlane(wave_search(a.s.n_seqs, place, first_tile));
        mine = kv4_rows(a.s.starts, b, a.s.rows);
        length = kv4_length(a.s.lengths, b);
        tile_of_rows = (int)max((int64_t)-1, place - first_tile(b));
    }
    const int rows = mine.count * G;                                   // tokens x query heads of the kv head
    const int64_t base64 = (int64_t)tile_of_rows * TILE;
    if (base64 < 0 || base64 >= rows) return;
    const int base = (int)base64 + (SHARE ? 0 : wave * 16 * QT);
    const int before = length - mine.count;                            // position of the sequence's first new token (< 0: it is not there)
    const int32_t* __restrict__ table = a.s.table + (int64_t)b * a.s.table_ld;

    // the tokens that each of this lane's rows sees, [from, to), and those that all / any of the wavefront's rows see: windows by the rows'
    // own tokens, which may lie behind the table, and no token behind the table
    const int places = kv4_places(a.s.max_pages, a.c.shift);
    auto end_of = [&](int i) { return a.q.causal ? before + i + 1 : length; };        // new token i's
    // (a row before token 0 has an end below 0, from which a wide window would pass 32 bits)
    auto start_of = [&](int i) { return a.q.window > 0 ? max(0, max(0, end_of(i)) - a.q.window) : 0; };
    int from[QT], to[QT];
    u4 qf[QT][D / 32];
    float qsum[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int rho = base + 16 * t + col;
        const bool there = rho < rows;
        const int i = there ? rho / G : 0, hq = there ? rho - i * G : 0;
        to[t] = there ? min(places, end_of(i)) : 0;
        from[t] = start_of(i);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) {
            u4 raw = {0, 0, 0, 0};
            if (there) {
                const T* src = static_cast<const T*>(a.q.q) + (int64_t)(mine.first + i) * a.q.q_row + (int64_t)(h * G + hq) * a.q.q_head + (D / 4) * g + 8 * k;
                __builtin_memcpy(&raw, src, 16);
            }
            T el[8];
            __builtin_memcpy(el, &raw, 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += (float)el[e];
            // channels e and e + 4 share a register, as the codes do
            u4 f;
            f[0] = __builtin_amdgcn_perm(raw[2], raw[0], 0x05040100u);
            f[1] = __builtin_amdgcn_perm(raw[2], raw[0], 0x07060302u);
            f[2] = __builtin_amdgcn_perm(raw[3], raw[1], 0x05040100u);
            f[3] = __builtin_amdgcn_perm(raw[3], raw[1], 0x07060302u);
            qf[t][k] = f;
        }
        qsum[t] = quarters_sum(sum);
    }
    // what any of the wavefront's rows sees, and what all of them see (rows that are not there may see what they like)
    const int row0 = min(base, rows - 1) / G, row1 = (min(base + 16 * QT, rows) - 1) / G;
    int any_to = base < rows ? max(0, min(places, end_of(row1))) : 0, all_to = min(places, end_of(row0));
    const int any_from = start_of(row0), all_from = start_of(row1);

    // this part's tokens, in tiles of 32; without SHARE the workgroup's rows, and `needed` those tiles that the wavefront's see
    int wg_from = any_from, wg_to = any_to;
    if constexpr (!SHARE) {
        const int first = (int)base64, final = min(first + TILE, rows) - 1;
        wg_to = max(0, min(places, end_of(final / G)));
        wg_from = start_of(first / G);
    }
    const int tile0 = wg_from / 32, tile1 = (wg_to + 31) / 32;
    const int per = (max(0, tile1 - tile0) + parts - 1) / parts;
    const int begin = tile0 + part * per, end = min(tile1, begin + per);

    f4 o[QT][M];
    float m[QT], l[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = NEG_MAX;
        l[t] = 0.f;
#pragma unroll
        for (int j = 0; j < M; ++j) o[t][j] = f4{0.f, 0.f, 0.f, 0.f};
    }

    // A lane works on the grids of one token; the eight it needs come from the lanes of its quarter.
    // The scores of 32 tokens, but for their scales.  key(i, k): the fragments
    auto scores = [&](uint32_t k_grid, f4 (&s)[QT][2], auto key) {
        const float kz = -(Frag<T>::OFFSET + (float)kv4_zero(k_grid));
        for8([&](auto e) {
            constexpr int E = decltype(e)::value;
#pragma unroll
            for (int t = 0; t < QT; ++t) s[t][E >> 2][E & 3] = from_lane<E>(kz) * qsum[t];
        });
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const u4 kf = key(i, k);
#pragma unroll
                for (int t = 0; t < QT; ++t) s[t][i] = Frag<T>::mfma(kf, qf[t][k], s[t][i]);
            }
    };
    // u: scores above the running maximum, in binary orders, which is raised where that is needed.  Returns whether all rows see all tokens.
    auto above = [&](int t0, const Grids& grids, const f4 (&s)[QT][2], float (&u)[QT][8]) {
        const float ka = __uint_as_float(grids.k & 0xffff0000u) * a.scale2, vlog = (float)(max((int)(grids.v >> 23), 127 + VALUE_FLOOR) - 127);
        float kas[8], most = -INFINITY;
        for8([&](auto e) { kas[decltype(e)::value] = from_lane<decltype(e)::value>(ka); });
        float vtop = fmaxf(vlog, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(vlog), 0xB1, 0xf, 0xf, true)));      // over the eight
        vtop = fmaxf(vtop, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(vtop), 0x4E, 0xf, 0xf, true)));
        vtop = fmaxf(vtop, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(vtop), 0x141, 0xf, 0xf, true)));
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) u[t][e] = fmaf(s[t][e >> 2][e & 3], kas[e], -m[t]);
        const bool whole = grids.first && grids.last && t0 >= all_from && t0 + 32 <= all_to;
        if (!whole) {
            const bool page = (g & 2) ? grids.last : grids.first;
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int tok = t0 + 8 * g + e;
                    if (tok < from[t] || tok >= to[t] || !page) u[t][e] = -INFINITY;
                }
        }
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, u[t][e]);
        // no P can pass 2^RAISE; where one might, the maximum is raised to what the tokens have
        if (__any(most + vtop > BIAS + RAISE)) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                float z = -INFINITY;
                for8([&](auto e) {
                    constexpr int E = decltype(e)::value;
                    const float log = from_lane<E>(vlog);              // (all lanes take part)
                    if (u[t][E] != -INFINITY) {
                        u[t][E] = s[t][E >> 2][E & 3] * kas[E];
                        z = fmaxf(z, u[t][E] + log);
                    }
                });
                const float up = fmaxf(m[t], quarters_max(z) - BIAS), f = __builtin_amdgcn_exp2f(m[t] - up);
#pragma unroll
                for (int e = 0; e < 8; ++e) u[t][e] -= up;
                m[t] = up;
                l[t] *= f;
#pragma unroll
                for (int j = 0; j < M; ++j) o[t][j] *= f;
            }
        }
        return whole;
    };
    // the weights times the values' scales, and their sums
    auto weigh = [&](uint32_t v_grid, const float (&u)[QT][8], f16x8 (&p)[QT]) {
        const float va = __uint_as_float(v_grid & 0xffff0000u) * (LIFT / BIAS2);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(u[t][e]);
            l[t] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            for8([&](auto e) { p[t][decltype(e)::value] = (f16_t)(w[decltype(e)::value] * from_lane<decltype(e)::value>(va)); });
        }
    };
    // nothing from tokens that are not seen, also where their values are NaN
    auto forget = [&](const float (&u)[QT][8], f16x8 (&p)[QT]) {
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (u[t][e] == -INFINITY) p[t][e] = (f16_t)0.f;
    };
    // value(u, n): the fragments
    auto add = [&](const f16x8 (&p)[QT], auto value) {
#pragma unroll
        for (int n = 0; n < M; ++n) {
            const u4 vf = value(n >> 2, n & 3);
#pragma unroll
            for (int t = 0; t < QT; ++t) o[t][n] = Frag<f16_t>::mfma(vf, __builtin_bit_cast(u4, p[t]), o[t][n]);
        }
    };
    PageRow row_of_pages{table};
    auto pages = [&](int tile) { return row_of_pages.pages(a.c, a.s.max_pages, tile * 32); };
    if constexpr (SHARE) {
        // the tokens of the next tile are on their way while a tile is attended to
        int tile = begin + wave;
        if (tile < end) {
            using X = Tokens<D>;
            X x0, x1;
            auto use = [&](X& x) {
                const Zeros z = value_zeros(x.grids.v, bits);
                uint32_t pair[4];
                f4 s[QT][2];
                float u[QT][8];
                f16x8 p[QT];
                scores(x.grids.k, s, [&](int i, int k) { return Frag<T>::codes(x.k[i][k], bits); });
                const bool whole = above(tile * 32, x.grids, s, u);
                weigh(x.grids.v, u, p);
                if (!whole) forget(u, p);
                add(p, [&](int w, int n) {
                    if (n == 0)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            pair[j] = __builtin_amdgcn_perm(x.v[2 * j + 1][w / 2], x.v[2 * j][w / 2], w & 1 ? 0x07060302u : 0x05040100u);
                    return value_fragment(pair, n, z, bits);
                });
            };
            load_tokens<D>(a.c, pages(tile), h, tile * 32, x0);
            for (;;) {
                if (tile + WAVES < end) load_tokens<D>(a.c, pages(tile + WAVES), h, (tile + WAVES) * 32, x1);
                use(x0);
                if ((tile += WAVES) >= end) break;
                if (tile + WAVES < end) load_tokens<D>(a.c, pages(tile + WAVES), h, (tile + WAVES) * 32, x0);
                use(x1);
                if ((tile += WAVES) >= end) break;
            }
        }
    } else if (begin < end) {
        // A stage is SUB tiles of 32 tokens.  4 / SUB wavefronts turn a tile's codes into fragments, each OF of K (numbers i D / 32 + k: one
        // i, adjacent words of a row) and as many of V (4 u + n: one u).
        constexpr int PER = WAVES / SUB, OF = M / PER, ROW = D / 2;
        const int sub = wave / PER, f0 = wave % PER * OF, final = end - 1;
        // Dim 128 has the registers to take the second tile's scores beside the first one's weights, and to read V's fragments ahead (A prompt
        // of 8192 tokens, 32 query heads: 671 us, 699 without; dim 64 would lose the third wavefront of a SIMD: 155 us, 133 without, for 4 of 2048).
        constexpr bool AHEAD = D == 128;
        // a stage may pass the end of the part
        any_to = min(any_to, end * 32);
        all_to = min(all_to, end * 32);
#pragma unroll
        for (int t = 0; t < QT; ++t) to[t] = min(to[t], end * 32);
        struct Raw { uint32_t k[OF]; uint32_t v[8]; Grids grids[SUB]; };  // v: four channels of a token (put together only when they are here)
        auto load = [&](int tile, Raw& x) {
            Where mine;
#pragma unroll
            for (int q = 0; q < SUB; ++q) {
                const int t = min(tile + q, final);
                const Where w = where(a.c, pages(t), h, t * 32);
                load_grids(a.c, w, x.grids[q]);
                if (q == 0 || q == sub) mine = w;
            }
            at_token(a.c, mine, col & 8, [&](int64_t row) {
                const unsigned at = (8 * (col >> 2) + (col & 3) + 4 * (f0 / (D / 32))) * ROW + (D / 8) * g + 4 * (f0 % (D / 32));
                __builtin_memcpy(x.k, __builtin_assume_aligned(a.c.k_codes + row * ROW + at, 4 * OF), sizeof x.k);
            });
            at_token(a.c, mine, g & 2, [&](int64_t row) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x.v[e] = *reinterpret_cast<const uint16_t*>(a.c.v_codes + row * ROW + (unsigned)((8 * g + e) * ROW + (D / 32) * col + 2 * (f0 >> 2)));
            });
        };
        auto stage = [&](int buf, const Raw& x) {
            u4* dst = &sh_f[buf][sub * 2 * M + f0][lane];
#pragma unroll
            for (int j = 0; j < OF; ++j) dst[j * 64] = Frag<T>::codes(x.k[j], bits);
            uint32_t grid = x.grids[0].v;
#pragma unroll
            for (int q = 1; q < SUB; ++q) grid = q == sub ? x.grids[q].v : grid;
            const Zeros z = value_zeros(grid, bits);
            // from channel 0 or (dim 64) 0 or 2 of the four on; 2 and 3 are a byte up
            uint32_t pair[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) pair[j] = (x.v[2 * j] | x.v[2 * j + 1] << 16) >> (OF < 4 && (f0 & 2) ? 8 : 0);
#pragma unroll
            for (int n = 0; n < OF; ++n) dst[(M + n) * 64] = value_fragment(pair, n, z, bits);
        };
        Raw raw;
        load(begin, raw);
        stage(0, raw);
        Grids grids[SUB];
#pragma unroll
        for (int q = 0; q < SUB; ++q) grids[q] = raw.grids[q];
        if (begin + SUB < end) load(begin + SUB, raw);
        for (int tile = begin; tile < end; tile += SUB) {
            const int buf = (tile - begin) / SUB & 1;
            // this stage's fragments are in LDS, and everybody is done with the other buffer
            __syncthreads();
            Grids next[SUB];
#pragma unroll
            for (int q = 0; q < SUB; ++q) next[q] = raw.grids[q];
            if (tile + SUB < end) stage(buf ^ 1, raw);
            if (tile + 2 * SUB < end) load(tile + 2 * SUB, raw);
            if (tile * 32 < any_to && (tile + SUB) * 32 > any_from) {
                auto key = [&](int q) { return [&, q](int i, int k) { return sh_f[buf][q * 2 * M + i * (D / 32) + k][lane]; }; };
                f4 s[AHEAD ? SUB : 1][QT][2];
                if (AHEAD) scores(grids[0].k, s[0], key(0));
#pragma unroll
                for (int q = 0; q < SUB; ++q) {
                    const int t0 = (tile + q) * 32;
                    if (!AHEAD && (t0 >= any_to || t0 + 32 <= any_from)) continue;
                    float u[QT][8];
                    f16x8 p[QT];
                    u4 vf[AHEAD ? M : 1];
                    if (!AHEAD) scores(grids[q].k, s[0], key(q));
                    const bool whole = above(t0, grids[q], s[AHEAD ? q : 0], u);
                    if (AHEAD && q + 1 < SUB) scores(grids[SUB - 1].k, s[SUB - 1], key(SUB - 1));
                    if (AHEAD) {
#pragma unroll
                        for (int n = 0; n < M; ++n) vf[n] = sh_f[buf][q * 2 * M + M + n][lane];
                        __builtin_amdgcn_sched_barrier(0x47E);         // (not to be read where they are used)
                    }
                    weigh(grids[q].v, u, p);
                    if (!whole) forget(u, p);
                    add(p, [&](int w, int n) { return AHEAD ? vf[AHEAD ? 4 * w + n : 0] : sh_f[buf][q * 2 * M + M + 4 * w + n][lane]; });
                }
            }
#pragma unroll
            for (int q = 0; q < SUB; ++q) grids[q] = next[q];
        }
    }

    // sums over the four lanes of a column
#pragma unroll
    for (int t = 0; t < QT; ++t) l[t] = quarters_sum(l[t]);

    // N channels from `ch` on of row `rho`: value(k) before the division by the sum
    auto finish = [&](int rho, int ch, auto channels, float mm, float ll, auto value) {
        constexpr int N = decltype(channels)::value;
        if (rho >= rows) return;
        const int i = rho / G, head = h * G + rho - i * G;
        const int64_t token = mine.first + i;
        if (parts > 1) {
            const int64_t at = ((int64_t)h * a.slots + index) * TILE + rho - base64;
            if (ch == 0) { a.part_ml[2 * at] = mm; a.part_ml[2 * at + 1] = ll; }
            f4* dst = reinterpret_cast<f4*>(a.part_o + at * D + ch);
#pragma unroll
            for (int j = 0; j < N / 4; ++j) dst[j] = f4{value(4 * j), value(4 * j + 1), value(4 * j + 2), value(4 * j + 3)};
            return;
        }
        const float inv = ll == 0.f ? 0.f : BIAS2 / LIFT / ll;                // a row that sees nothing is 0
        T out[N];
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = (T)(value(k) * inv);
        __builtin_memcpy(static_cast<T*>(a.q.out) + token * a.q.out_row + (int64_t)head * a.q.out_head + ch, out, sizeof out);
        if (a.q.lse && ch == 0) a.q.lse[token * a.heads_q + head] = ll == 0.f ? -INFINITY : LN2 * mm + logf(ll);
    };
    // value k of this lane's dim / 4 channels: channel (dim / 4) g + (dim / 16) i + n is o[n][i]
    if constexpr (!SHARE) {
#pragma unroll
        for (int t = 0; t < QT; ++t)
            finish(base + 16 * t + col, (D / 4) * g, std::integral_constant<int, D / 4>(), m[t], l[t], [&](int k) { return o[t][k % M][k / M]; });
    } else {
        // the wavefronts' results meet in LDS; each thread then has dim / 16 channels of a row
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            f4* dst = reinterpret_cast<f4*>(&sh_o[wave][(16 * t + col) * (D + 4) + (D / 4) * g]);
#pragma unroll
            for (int k = 0; k < D / 4; k += 4)
                dst[k / 4] = f4{o[t][k % M][k / M], o[t][(k + 1) % M][(k + 1) / M], o[t][(k + 2) % M][(k + 2) / M], o[t][(k + 3) % M][(k + 3) / M]};
            if (g == 0) { sh_ml[wave][2 * (16 * t + col)] = m[t]; sh_ml[wave][2 * (16 * t + col) + 1] = l[t]; }
        }
        __syncthreads();
        const int ch = (threadIdx.x & 15) * (D / 16);
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int row = 16 * t + (threadIdx.x >> 4);
            float mm = NEG_MAX, w[WAVES], ll = 0.f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) mm = fmaxf(mm, sh_ml[k][2 * row]);
#pragma unroll
            for (int k = 0; k < WAVES; ++k) {
                w[k] = __builtin_amdgcn_exp2f(sh_ml[k][2 * row] - mm);
                ll += w[k] * sh_ml[k][2 * row + 1];
            }
            float sum[D / 16];
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                sum[c] = 0.f;
#pragma unroll
                for (int k = 0; k < WAVES; ++k) sum[c] += w[k] * sh_o[k][row * (D + 4) + ch + c];
            }
            finish(base + row, ch, std::integral_constant<int, D / 16>(), mm, ll, [&](int k) { return sum[k]; });
        }
    }
}

// The parts of a row joined: one wavefront per row and query head.  Parts whose rows saw nothing have a sum of 0.  (1024 rows: 4 us, most of
// which is the launch; finding the split again here, instead of reading it, took 2 more.)
template <class T, int D>
__global__ __launch_bounds__(256) void kv4_join_kernel(AttnArgs a)
{
    constexpr int N = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int token = __builtin_amdgcn_readfirstlane((int)(item / a.heads_q));
    const int head = __builtin_amdgcn_readfirstlane((int)(item - (int64_t)token * a.heads_q));
    if (token >= a.s.rows) return;
    const int b = __builtin_amdgcn_readfirstlane(wave_search(a.s.n_seqs, token, [&](int i) { return (int64_t)kv4_rows(a.s.starts, i, a.s.rows).first; }));
    const Kv4Rows mine = kv4_rows(a.s.starts, b, a.s.rows);
    if (token < mine.first || token >= mine.first + mine.count) return;       // a row of no sequence
    const int first = __builtin_amdgcn_readfirstlane(a.seqs[b].x), parts = __builtin_amdgcn_readfirstlane(a.seqs[b].y);
    if (parts == 1) return;                                                   // its results are there
    const int G = a.q.group, h = head / G, rho = (token - mine.first) * G + head - h * G, tile = rho / a.tile;
    if (first + (tile + 1) * parts > a.slots) return;                         // (starts out of order)
    // part p's sums
    const int64_t at0 = ((int64_t)h * a.slots + first + tile * parts) * a.tile + rho - tile * a.tile, stride = a.tile;
    float m = NEG_MAX, l = 0.f;
    if (lane < parts) { m = a.part_ml[2 * (at0 + lane * stride)]; l = a.part_ml[2 * (at0 + lane * stride) + 1]; }
    float top = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    const float w = __builtin_amdgcn_exp2f(m - top);
    float sum = w * l;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    float y[N];
#pragma unroll
    for (int c = 0; c < N; ++c) y[c] = 0.f;
    // four parts' loads in flight; those behind the last are none (the last one's, times 0)
    for (int p0 = 0; p0 < parts; p0 += 4) {
        float v[4][N], wp[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = min(p0 + k, parts - 1);
            wp[k] = p0 + k < parts ? __shfl(w, p) : 0.f;
            __builtin_memcpy(v[k], a.part_o + (at0 + p * stride) * D + N * lane, sizeof v[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int c = 0; c < N; ++c) y[c] += wp[k] * v[k][c];
    }
    const float inv = sum == 0.f ? 0.f : BIAS2 / LIFT / sum;
    T out[N];
#pragma unroll
    for (int c = 0; c < N; ++c) out[c] = (T)(y[c] * inv);
    __builtin_memcpy(static_cast<T*>(a.q.out) + (int64_t)token * a.q.out_row + (int64_t)head * a.q.out_head + N * lane, out, sizeof out);
    if (a.q.lse && lane == 0) a.q.lse[(int64_t)token * a.heads_q + head] = sum == 0.f ? -INFINITY : LN2 * top + logf(sum);
}

Kv4Plan kv4_attention_plan(int cus, int dim, int heads, int group, int n_seqs, int64_t rows, int64_t longest)
{
    // The form goes by the average: the host does not know a sequence's rows.  What it was chosen by are calls of sequences alike; where prompts
    // and single tokens share a call, the one or the other runs in a form that is not its own (results are the same to rounding).
    Kv4Plan p;
    const int64_t each = n_seqs > 0 ? (rows * group + n_seqs - 1) / n_seqs : 0;     // rows of a sequence and kv head, on average
    p.share = each <= (dim == 256 ? 16 : 32);
    p.tile = p.share ? (each <= 16 ? 16 : 32) : (dim == 256 ? 64 : 128);
    p.tiles = rows * group / p.tile + n_seqs;
    // Sequences are split where there are fewer tiles of rows than the chip holds workgroups at a time, by their registers and LDS.  (Dim 128,
    // 8 heads: 128 sequences of 1024 tokens 38 us, 46 if they are split; 96 of up to 2048 39, 53; 128 of up to 4096 93, 99.)
    const int64_t full = (p.share && p.tile == 16 ? (dim == 64 ? 4 : dim == 128 ? 3 : 2) : 2) * (int64_t)cus / heads;
    p.slots = 0;
    if (longest > KV4_UNSPLIT && n_seqs <= KV4_SPLIT_SEQS && p.tiles < full)
        p.slots = (int)std::max(full, p.tiles + p.tiles / 2 + 1);
    return p;
}

int64_t kv4_attention_workspace(const Kv4Plan& p, int dim, int heads)
{
    return p.slots ? (int64_t)heads * p.slots * p.tile * (dim + 2) * (int64_t)sizeof(float) + KV4_SPLIT_SEQS * (int64_t)sizeof(int2) : 0;
}

template <class T, int D>
static hipError_t attention_of(hipStream_t st, const Kv4Plan& p, const AttnArgs& a)
{
    const dim3 grid((unsigned)((p.slots ? p.slots : p.tiles) * a.c.heads)), block(256);
    if (p.share && p.tile == 16) hipLaunchKernelGGL((kv4_attention_kernel<T, D, 1, true>), grid, block, 0, st, a);
    else if constexpr (D == 256) hipLaunchKernelGGL((kv4_attention_kernel<T, D, 1, false>), grid, block, 0, st, a);
    else if (p.share) hipLaunchKernelGGL((kv4_attention_kernel<T, D, 2, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv4_attention_kernel<T, D, 2, false>), grid, block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.slots) return e;
    const int64_t items = (int64_t)a.s.rows * a.heads_q;
    hipLaunchKernelGGL((kv4_join_kernel<T, D>), dim3((unsigned)((items + 3) / 4)), block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv4_attention(hipStream_t st, const Kv4Plan& p, const Kv4View& c, const Kv4Seqs& s, int type, const Kv4Query& q, float* work)
{
    AttnArgs a{c, s, q, c.heads * q.group, p.tile, p.slots, q.scale * LOG2E, work, nullptr, nullptr};
    if (work) {
        a.part_ml = work + (int64_t)c.heads * p.slots * p.tile * c.dim;
        a.seqs = reinterpret_cast<int2*>(a.part_ml + (int64_t)c.heads * p.slots * p.tile * 2);
    }
    if (type == FOBQ_BF16)
        return c.dim == 64 ? attention_of<bf16_t, 64>(st, p, a) : c.dim == 128 ? attention_of<bf16_t, 128>(st, p, a) : attention_of<bf16_t, 256>(st, p, a);
    return c.dim == 64 ? attention_of<f16_t, 64>(st, p, a) : c.dim == 128 ? attention_of<f16_t, 128>(st, p, a) : attention_of<f16_t, 256>(st, p, a);
}

}  // namespace fobq
