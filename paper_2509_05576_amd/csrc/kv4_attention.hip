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
// fp16 weights and the range of V: m is the running maximum of S + log2 scale_v (its whole part), not of S, so that a row's largest weights
// are near 1 whatever the size of the values.  The sum of the softmax has the same m and takes any size in fp32; values below 2^-88
// count as that large there, which keeps it finite.
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
constexpr int VALUE_FLOOR = -88;
constexpr float RAISE = 8.f;            // binary orders of magnitude that a score may exceed the running maximum by
constexpr int KV4_PART = 256;           // tokens of a part at least: eight tiles, two for each wavefront that shares the rows
constexpr int KV4_MAX_PARTS = 64;       // a lane each where they are joined
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;

struct AttnArgs {
    Kv4View c; Kv4Seqs s; Kv4Query q;
    int parts, heads_q;
    float scale2;          // scale * log2(e)
    float* part_o;         // parts x rows x query heads x dim
    float* part_ml;        // the same without dim: maximum (in binary orders) and sum
};

template <class T> struct Frag;
template <> struct Frag<bf16_t> {
    static __device__ __forceinline__ f4 mfma(u4 a, u4 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static constexpr float OFFSET = 128.f;
    // 8 codes as 128 + code: register j has codes j and j + 4
    static __device__ __forceinline__ u4 codes(uint32_t w)
    {
        u4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = (w >> (4 * j) & 0x000f000fu) | 0x43004300u;
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
    static __device__ __forceinline__ u4 codes(uint32_t w)
    {
        u4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = j < 2 ? w : w >> 8;
            const h2 low = __builtin_bit_cast(h2, (x & 0x000f000fu) | 0x64006400u), high = __builtin_bit_cast(h2, (x & 0x00f000f0u) | 0x64006400u);
            const h2 v = j & 1 ? __builtin_elementwise_fma(high, h2{(f16_t)0.0625f, (f16_t)0.0625f}, h2{(f16_t)-64.f, (f16_t)-64.f})
                               : low + h2{(f16_t)-1024.f, (f16_t)-1024.f};
            r[j] = __builtin_bit_cast(uint32_t, v);
        }
        return r;
    }
};

// the four lanes of a column, a quarter of the wavefront apart
__device__ __forceinline__ float quarters_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quarters_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// 32 tokens' codes and grids of one head, as a lane uses them
template <int D> struct Tokens {
    static constexpr int K = D / 32, V = D / 128 > 0 ? D / 128 : 1;   // words of a K row, words of a V row (dim 64: half a word)
    uint32_t k[2][K];
    uint32_t v[8][V];
    u4 kg[2], vg[2];
    bool ok0, ok1;             // whether the first and the last 16 tokens lie on a page
};

template <int D>
__device__ __forceinline__ void load_tokens(const Kv4View& c, const int32_t* __restrict__ table, int max_pages, int h, int t0, Tokens<D>& x)
{
    constexpr int ROW = D / 2;
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int p0 = kv4_page(table, max_pages, c.pages, c.shift, t0), p1 = kv4_page(table, max_pages, c.pages, c.shift, t0 + 16);
    x.ok0 = p0 >= 0;
    x.ok1 = p1 >= 0;
    // tokens on no page: page 0 is read in their place, and masked
    const int mask = (1 << c.shift) - 1;
    const int64_t row0 = ((((int64_t)(p0 < 0 ? 0 : p0)) * c.heads + h) << c.shift) + (t0 & mask);
    const int64_t row1 = ((((int64_t)(p1 < 0 ? 0 : p1)) * c.heads + h) << c.shift) + ((t0 + 16) & mask) - 16;
    // K: row r of instruction i is token 8 (r / 4) + 4 i + r % 4
    const int64_t kr = ((r & 8) ? row1 : row0) + 8 * (r >> 2) + (r & 3);
#pragma unroll
    for (int i = 0; i < 2; ++i) __builtin_memcpy(x.k[i], __builtin_assume_aligned(c.k_codes + (kr + 4 * i) * ROW + 4 * Tokens<D>::K * g, D == 64 ? 8 : 16), sizeof x.k[i]);
    const int64_t vr = ((g & 2) ? row1 : row0) + 8 * g;
    const uint8_t* __restrict__ v = c.v_codes + vr * ROW + (D / 32) * r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (D == 64) x.v[e][0] = *reinterpret_cast<const uint16_t*>(v + e * ROW);
        else __builtin_memcpy(x.v[e], __builtin_assume_aligned(v + e * ROW, 4 * Tokens<D>::V), sizeof x.v[e]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x.kg[i] = *reinterpret_cast<const u4*>(c.k_grids + vr + 4 * i);
        x.vg[i] = *reinterpret_cast<const u4*>(c.v_grids + vr + 4 * i);
    }
}

// WAVES wavefronts; each has QT x 16 query rows: its own ones, or (SHARE) the workgroup's, of whose tokens it takes every WAVES-th tile.
template <class T, int D, int QT, bool SHARE>
__global__ __launch_bounds__(256, SHARE ? 2 : 2) void kv4_attention_kernel(AttnArgs a)
{
    constexpr int WAVES = 4, M = D / 16, TILE = 16 * QT * (SHARE ? 1 : WAVES);
    using X = Tokens<D>;
    __shared__ float sh_o[SHARE ? WAVES : 1][SHARE ? 16 * QT * (D + 4) : 1];
    __shared__ float sh_ml[SHARE ? WAVES : 1][SHARE ? 16 * QT * 2 : 1];

    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int G = a.q.group;

    // the sequence and the rows of this workgroup: sequence b's tiles begin at floor(first row * G / TILE) + b, which leaves room for
    // every sequence's last, partial tile
    auto first_tile = [&](int b) { return (int64_t)kv4_rows(a.s.starts, b, a.s.rows).first * G / TILE + b; };
    const int b = __builtin_amdgcn_readfirstlane(wave_search(a.s.n_seqs, (int64_t)blockIdx.x, first_tile));
    const Kv4Rows mine = kv4_rows(a.s.starts, b, a.s.rows);
    const int rows = mine.count * G;                                   // tokens x query heads of the kv head
    const int64_t base64 = ((int64_t)blockIdx.x - first_tile(b)) * TILE;
    if (base64 < 0 || base64 >= rows) return;
    const int base = (int)base64 + (SHARE ? 0 : wave * 16 * QT);
    const int h = blockIdx.y, part = blockIdx.z;
    const int length = kv4_length(a.s.lengths, b, a.s.max_pages, a.c.shift);
    const int before = length - mine.count;                            // position of the sequence's first new token (< 0: it is not there)
    const int32_t* __restrict__ table = a.s.table + (int64_t)b * a.s.table_ld;

    // the tokens that each of this lane's rows sees, [from, to), and those that all / any of the wavefront's rows see
    int from[QT], to[QT];
    u4 qf[QT][D / 32];
    float qsum[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int rho = base + 16 * t + col;
        const bool there = rho < rows;
        const int i = there ? rho / G : 0, hq = there ? rho - i * G : 0;
        to[t] = there ? (a.q.causal ? before + i + 1 : length) : 0;
        from[t] = a.q.window > 0 ? max(0, to[t] - a.q.window) : 0;
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
    const int last = max(base, min(base + 16 * QT, rows) - 1);
    const int to0 = a.q.causal ? before + base / G + 1 : length, to1 = a.q.causal ? before + last / G + 1 : length;
    const int any_to = base < rows ? max(0, to1) : 0, all_to = to0;
    const int any_from = a.q.window > 0 ? max(0, to0 - a.q.window) : 0, all_from = a.q.window > 0 ? max(0, to1 - a.q.window) : 0;

    // this part's tokens, in tiles of 32
    const int tile0 = any_from / 32, tile1 = (any_to + 31) / 32;
    const int per = max((max(0, tile1 - tile0) + a.parts - 1) / a.parts, KV4_PART / 32);
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

    const int step = SHARE ? WAVES : 1;
    int tile = begin + (SHARE ? wave : 0);
    X x;
    if (tile < end) load_tokens<D>(a.c, table, a.s.max_pages, h, tile * 32, x);
    for (; tile < end; tile += step) {
        X next;
        if (tile + step < end) load_tokens<D>(a.c, table, a.s.max_pages, h, (tile + step) * 32, next);
        const int t0 = tile * 32;

        // scores
        f4 s[QT][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int t = 0; t < QT; ++t) s[t][i] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const u4 kf = Frag<T>::codes(x.k[i][k]);
#pragma unroll
                for (int t = 0; t < QT; ++t) s[t][i] = Frag<T>::mfma(kf, qf[t][k], s[t][i]);
            }
        }
        const bool edge = !(x.ok0 && x.ok1 && t0 >= all_from && t0 + 32 <= all_to);
        float ka[8], kz[8], va[8], vlog[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t w = x.kg[e >> 2][e & 3], v = x.vg[e >> 2][e & 3];
            ka[e] = __uint_as_float(w & 0xffff0000u) * a.scale2;
            kz[e] = -(Frag<T>::OFFSET + (float)kv4_zero(w));
            va[e] = __uint_as_float(v & 0xffff0000u);
            vlog[e] = (float)max((int)(v >> 23) - 127, VALUE_FLOOR);
        }
        u4 pf[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(kz[e], qsum[t], s[t][e >> 2][e & 3]) * ka[e];
            if (edge) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int tok = t0 + 8 * g + e;
                    if (tok < from[t] || tok >= to[t] || !((g & 2) ? x.ok1 : x.ok0)) y[e] = -INFINITY;
                }
            }
            float top = y[0] + vlog[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, y[e] + vlog[e]);
            top = quarters_max(top);
            if (__any(top > m[t] + RAISE)) {
                const float up = fmaxf(m[t], top), f = __builtin_amdgcn_exp2f(m[t] - up);
                m[t] = up;
                l[t] *= f;
#pragma unroll
                for (int j = 0; j < M; ++j) o[t][j] *= f;
            }
            f16x8 p;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __builtin_amdgcn_exp2f(y[e] - m[t]);
                sum += w;
                p[e] = (f16_t)(w * va[e]);
            }
            if (edge) {
                // also where the token's values are NaN
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (y[e] == -INFINITY) p[e] = (f16_t)0.f;
            }
            l[t] += sum;
            pf[t] = __builtin_bit_cast(u4, p);
        }
        // values: 8 tokens x (D / 16) codes of this lane, four channels (16 bits) at a time
        h2 off_low[4], off_high[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t z = kv4_zero(x.vg[j >> 1][2 * (j & 1)]) | kv4_zero(x.vg[j >> 1][2 * (j & 1) + 1]) << 16;
            off_low[j] = __builtin_bit_cast(h2, z | 0x64006400u);              // 1024 + zero
            off_high[j] = __builtin_bit_cast(h2, z << 4 | 0x54005400u);        // 64 + zero
        }
#pragma unroll
        for (int u = 0; u < D / 64; ++u) {
            uint32_t pair[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                pair[j] = __builtin_amdgcn_perm(x.v[2 * j + 1][u / 2], x.v[2 * j][u / 2], u & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                u4 vf;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = n < 2 ? pair[j] : pair[j] >> 8;
                    const h2 v = n & 1 ? __builtin_elementwise_fma(__builtin_bit_cast(h2, (w & 0x00f000f0u) | 0x64006400u),
                                                                  h2{(f16_t)0.0625f, (f16_t)0.0625f}, -off_high[j])
                                       : __builtin_bit_cast(h2, (w & 0x000f000fu) | 0x64006400u) - off_low[j];
                    vf[j] = __builtin_bit_cast(uint32_t, v);
                }
#pragma unroll
                for (int t = 0; t < QT; ++t) o[t][4 * u + n] = Frag<f16_t>::mfma(vf, pf[t], o[t][4 * u + n]);
            }
        }
        x = next;
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
        if (a.parts > 1) {
            const int64_t at = ((int64_t)part * a.s.rows + token) * a.heads_q + head;
            if (ch == 0) { a.part_ml[2 * at] = mm; a.part_ml[2 * at + 1] = ll; }
            f4* dst = reinterpret_cast<f4*>(a.part_o + at * D + ch);
#pragma unroll
            for (int j = 0; j < N / 4; ++j) dst[j] = f4{value(4 * j), value(4 * j + 1), value(4 * j + 2), value(4 * j + 3)};
            return;
        }
        const float inv = ll == 0.f ? 0.f : 1.f / ll;                  // a row that sees nothing is 0
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

// The parts of a row joined: one wavefront per row and query head.  Parts whose rows saw nothing have a sum of 0.
template <class T, int D>
__global__ __launch_bounds__(256) void kv4_join_kernel(AttnArgs a)
{
    constexpr int N = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t token = item / a.heads_q;
    const int head = (int)(item - token * a.heads_q);
    const Kv4Rows first = kv4_rows(a.s.starts, 0, a.s.rows), last = kv4_rows(a.s.starts, a.s.n_seqs - 1, a.s.rows);
    if (token < first.first || token >= last.first + last.count) return;      // a row of no sequence
    const int64_t stride = (int64_t)a.s.rows * a.heads_q, at = token * a.heads_q + head;
    float m = NEG_MAX, l = 0.f;
    if (lane < a.parts) { m = a.part_ml[2 * (lane * stride + at)]; l = a.part_ml[2 * (lane * stride + at) + 1]; }
    float top = m;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    const float w = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top);
    float sum = w * l;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    float y[N];
#pragma unroll
    for (int c = 0; c < N; ++c) y[c] = 0.f;
    // four parts' loads in flight; those behind the last, and those that saw nothing, are none
    for (int p0 = 0; p0 < a.parts; p0 += 4) {
        float v[4][N], wp[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = min(p0 + k, a.parts - 1);
            wp[k] = p0 + k < a.parts ? __shfl(w, p) : 0.f;
            __builtin_memcpy(v[k], a.part_o + (p * stride + at) * D + N * lane, sizeof v[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int c = 0; c < N; ++c) y[c] += wp[k] == 0.f ? 0.f : wp[k] * v[k][c];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T out[N];
#pragma unroll
    for (int c = 0; c < N; ++c) out[c] = (T)(y[c] * inv);
    __builtin_memcpy(static_cast<T*>(a.q.out) + token * a.q.out_row + (int64_t)head * a.q.out_head + N * lane, out, sizeof out);
    if (a.q.lse && lane == 0) a.q.lse[at] = sum == 0.f ? -INFINITY : LN2 * top + logf(sum);
}

Kv4Plan kv4_attention_plan(int cus, int dim, int heads, int group, int n_seqs, int64_t rows, int64_t longest)
{
    Kv4Plan p;
    const int64_t each = n_seqs > 0 ? (rows * group + n_seqs - 1) / n_seqs : 0;     // rows of a sequence and kv head, on average
    p.share = each <= (dim == 256 ? 16 : 32);
    p.tile = p.share ? (each <= 16 ? 16 : 32) : (dim == 256 ? 64 : 128);
    p.tiles = rows * group / p.tile + n_seqs;
    const int64_t have = std::max<int64_t>(1, p.tiles * heads);
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(KV4_MAX_PARTS, (longest + KV4_PART - 1) / KV4_PART));
    p.parts = (int)std::min<int64_t>(most, std::max<int64_t>(1, (4 * (int64_t)cus + have - 1) / have));
    return p;
}

int64_t kv4_attention_workspace(const Kv4Plan& p, int dim, int heads, int group, int64_t rows)
{
    return p.parts > 1 ? p.parts * rows * heads * group * (dim + 2) * (int64_t)sizeof(float) : 0;
}

template <class T, int D>
static hipError_t attention_of(hipStream_t st, const Kv4Plan& p, const AttnArgs& a)
{
    const dim3 grid((unsigned)p.tiles, (unsigned)a.c.heads, (unsigned)p.parts), block(256);
    if (p.share && p.tile == 16) hipLaunchKernelGGL((kv4_attention_kernel<T, D, 1, true>), grid, block, 0, st, a);
    else if constexpr (D == 256) hipLaunchKernelGGL((kv4_attention_kernel<T, D, 1, false>), grid, block, 0, st, a);
    else if (p.share) hipLaunchKernelGGL((kv4_attention_kernel<T, D, 2, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv4_attention_kernel<T, D, 2, false>), grid, block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    const int64_t items = (int64_t)a.s.rows * a.heads_q;
    hipLaunchKernelGGL((kv4_join_kernel<T, D>), dim3((unsigned)((items + 3) / 4)), block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_kv4_attention(hipStream_t st, const Kv4Plan& p, const Kv4View& c, const Kv4Seqs& s, int type, const Kv4Query& q, float* work)
{
    AttnArgs a{c, s, q, p.parts, c.heads * q.group, q.scale * LOG2E, work, work ? work + (int64_t)p.parts * s.rows * c.heads * q.group * c.dim : nullptr};
    if (type == FOBQ_BF16)
        return c.dim == 64 ? attention_of<bf16_t, 64>(st, p, a) : c.dim == 128 ? attention_of<bf16_t, 128>(st, p, a) : attention_of<bf16_t, 256>(st, p, a);
    return c.dim == 64 ? attention_of<f16_t, 64>(st, p, a) : c.dim == 128 ? attention_of<f16_t, 128>(st, p, a) : attention_of<f16_t, 256>(st, p, a);
}

}  // namespace fobq
