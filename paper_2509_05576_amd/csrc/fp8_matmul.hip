// Product of two matrices in 8-bit floating point with a scale for each block of 128 columns:
//   Y[m][n] = sum_kb sa[kb][m] sb[kb][n / per] sum_{k in block kb} A[m][k] B[n][k]
// The outer sum is a multiply-add per value and block on the vector units, in fp32: acc += (sa sb) * part.  The inner one is
//   one 16x16x128 matrix instruction on 8-bit operands (its own scales at 1) for results in 16 bits.  That instruction adds the products
//     of eight neighbouring k's to 13 bits below the largest of them before its fp32 sums (measured: a product of 2^-14 of the largest is
//     lost, from another eight it is kept to 2^-23): 1.5e-5 of a block's result on Gaussian values, 5.5e-5 where they spread over
//     orders of magnitude, against the 2e-3 and 2.4e-4 that rounding to bf16 and fp16 leaves;
//   EXACT: four 16x16x32 instructions on the values as fp16, which holds both 8-bit types exactly (6e-8 with the same inputs), at
//     half the rate: for results in 32 bits.
//
// The instruction's rows are rows of B (outputs n), its columns rows of A (inputs m): a lane's four results are four consecutive n of
// one m, so sa is one value per lane and with a scale per 128 rows of B sb is the same for the whole wavefront.
//
// Tiles of both matrices are copied straight into LDS, 128 bytes a row, the 16-byte pieces of row r at places p ^ (r / 2 % 8): the 16
// rows that the lanes of a quarter read at once then lie in all 64 banks.  Which eight k's a lane holds does not matter, as both
// operands have the same.
#include "lowbit.h"

#include <algorithm>

namespace fobq {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));

struct MatmulArgs {
    Fp8View a, b;
    void* y; int type; int64_t ldy;
    float* work;                 // parts > 1: parts x m x n
    int parts, per_part;         // blocks of a part
};

// the matrix instruction's names of the types (fobq_fp8): 0 e4m3, 1 e5m2
template <int FB, int FA>
__device__ __forceinline__ f4 mfma_block(i8v b, i8v a)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, f4{0.f, 0.f, 0.f, 0.f}, FB, FA, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
}

// 4 values as fp16
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
template <int F>
__device__ __forceinline__ h2 as_fp16(int w, bool high)
{
    if constexpr (F == FOBQ_E4M3) return high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
    else return __builtin_bit_cast(h2, __builtin_amdgcn_perm(0u, (uint32_t)w, high ? 0x030c020cu : 0x010c000cu));   // e5m2 is fp16 without its last byte
}
template <int F> struct Block16 { h8 part[4]; };
template <int F>
__device__ __forceinline__ Block16<F> as_fp16(i8v x)
{
    Block16<F> b;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const h2 v0 = as_fp16<F>(x[2 * p], false), v1 = as_fp16<F>(x[2 * p], true), v2 = as_fp16<F>(x[2 * p + 1], false), v3 = as_fp16<F>(x[2 * p + 1], true);
        b.part[p] = h8{v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
    }
    return b;
}
template <int FB, int FA>
__device__ __forceinline__ f4 mfma_block(const Block16<FB>& b, const Block16<FA>& a)
{
    f4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < 4; ++p) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(b.part[p], a.part[p], c, 0, 0, 0);
    return c;
}
template <bool EXACT, int F>
__device__ __forceinline__ auto operand(i8v x)
{
    if constexpr (EXACT) return as_fp16<F>(x);
    else return x;
}

__device__ __forceinline__ void copy16(const void* src, void* lds_base)
{
    __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)src, (void __attribute__((address_space(3)))*)lds_base, 16, 0, 0);
}

__device__ __forceinline__ int swizzle(int row, int piece) { return piece ^ (row >> 1 & 7); }

// four consecutive n of row m
__device__ __forceinline__ void put4(const MatmulArgs& g, int part, int m, int n, f4 v)
{
    const int left = g.b.rows - n;
    if (g.parts > 1) {
        float* dst = g.work + ((int64_t)part * g.a.rows + m) * g.b.rows + n;
        if (left >= 4) __builtin_memcpy(dst, &v, 16);
        else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < left) dst[i] = v[i];
        }
        return;
    }
    auto out = [&](auto zero) {
        using T = decltype(zero);
        T* dst = static_cast<T*>(g.y) + (int64_t)m * g.ldy + n;
        T t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = (T)v[i];
        if (left >= 4) __builtin_memcpy(dst, t, sizeof t);
        else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < left) dst[i] = t[i];
        }
    };
    if (g.type == FOBQ_F32) out(0.f);
    else if (g.type == FOBQ_BF16) out((bf16_t)0.f);
    else out((f16_t)0.f);
}

// TM x TN outputs by WM x WN wavefronts.  FA, FB: the types of A and B; PER: rows of B to a scale.
template <int TM, int TN, int WM, int WN, int FA, int FB, int PER, bool EXACT>
__global__ __launch_bounds__(64 * WM * WN) void fp8_matmul_kernel(MatmulArgs g)
{
    constexpr int THREADS = 64 * WM * WN, SM = TM / WM / 16, SN = TN / WN / 16;
    __shared__ __attribute__((aligned(16))) uint8_t sh[2][(TM + TN) * 128];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, c = lane & 15;
    const int wm = wave / WN, wn = wave % WN;
    const int M = g.a.rows, N = g.b.rows, K = g.a.cols, blocks = (K + 127) / 128;
    const int m0 = blockIdx.x * TM, n0 = blockIdx.y * TN, part = blockIdx.z;
    const int kb0 = part * g.per_part, kb1 = min(blocks, kb0 + g.per_part);

    // pieces of a step's tiles, 16 bytes a thread: rows of A, then rows of B; rows behind the last are the last again
    constexpr int PIECES = (TM + TN) * 8 / THREADS;
    static_assert((TM * 8) % THREADS == 0 && (TN * 8) % THREADS == 0, "whole wavefronts of pieces");
    auto source = [&](int i, int kb) -> const uint8_t* {
        const int piece = i * THREADS + threadIdx.x, row = piece >> 3, k = swizzle(row, piece & 7) * 16;
        return row < TM ? g.a.values + (int64_t)min(m0 + row, M - 1) * g.a.ld + (int64_t)kb * 128 + k
                        : g.b.values + (int64_t)min(n0 + row - TM, N - 1) * g.b.ld + (int64_t)kb * 128 + k;
    };
    auto fetch = [&](int buf, int kb) {
        if (kb * 128 + 128 <= K) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) copy16(source(i, kb), &sh[buf][(i * THREADS + wave * 64) * 16]);
        } else {
            // the last block of columns is not whole: what is behind it counts as zero, whatever the rows hold there
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int piece = i * THREADS + threadIdx.x, row = piece >> 3, k = kb * 128 + swizzle(row, piece & 7) * 16;
                uint32_t w[4] = {0, 0, 0, 0};
                if (k < K) {
                    __builtin_memcpy(w, __builtin_assume_aligned(source(i, kb), 16), 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int have = K - k - 4 * j;
                        w[j] &= have >= 4 ? 0xffffffffu : have <= 0 ? 0u : (1u << (8 * have)) - 1;
                    }
                }
                __builtin_memcpy(__builtin_assume_aligned(&sh[buf][piece * 16], 16), w, 16);
            }
        }
    };
    auto fragment = [&](int buf, int row) {
        const uint8_t* p = &sh[buf][row * 128];
        const i4 lo = *reinterpret_cast<const i4*>(p + swizzle(row, 2 * q) * 16), hi = *reinterpret_cast<const i4*>(p + swizzle(row, 2 * q + 1) * 16);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f4 acc[SM][SN];
#pragma unroll
    for (int i = 0; i < SM; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    const int wm0 = wm * (TM / WM), wn0 = wn * (TN / WN);
    if (kb0 < kb1) fetch(0, kb0);
    for (int kb = kb0; kb < kb1; ++kb) {
        const int buf = (kb - kb0) & 1;
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (kb + 1 < kb1) fetch(buf ^ 1, kb + 1);
        float sa[SM];
        f4 sb[PER == 1 ? SN : 1];
#pragma unroll
        for (int i = 0; i < SM; ++i) sa[i] = g.a.scales[kb * g.a.ld_scales + min(m0 + wm0 + 16 * i + c, M - 1)];
        if constexpr (PER == 1) {
#pragma unroll
            for (int j = 0; j < SN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sb[j][e] = g.b.scales[kb * g.b.ld_scales + min(n0 + wn0 + 16 * j + 4 * q + e, N - 1)];
        } else {
            const float s = g.b.scales[kb * g.b.ld_scales + min(n0 + wn0, N - 1) / 128];
#pragma unroll
            for (int i = 0; i < SM; ++i) sa[i] *= s;
        }
        decltype(operand<EXACT, FB>(i8v())) bf[SN];
#pragma unroll
        for (int j = 0; j < SN; ++j) bf[j] = operand<EXACT, FB>(fragment(buf, TM + wn0 + 16 * j + c));
#pragma unroll
        for (int i = 0; i < SM; ++i) {
            const auto af = operand<EXACT, FA>(fragment(buf, wm0 + 16 * i + c));
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                f4 p = mfma_block<FB, FA>(bf[j], af);
                if constexpr (PER == 1) p *= sb[j];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], sa[i], acc[i][j][e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < SM; ++i) {
        const int m = m0 + wm0 + 16 * i + c;
        if (m < M)
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                const int n = n0 + wn0 + 16 * j + 4 * q;
                if (n < N) put4(g, part, m, n, acc[i][j]);
            }
    }
}

// the parts of a product, added in their order; four values a thread
__global__ __launch_bounds__(256) void fp8_matmul_join_kernel(MatmulArgs g)
{
    const int64_t quads = (g.b.rows + 3) / 4, item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = item / quads;
    const int n = (int)(item - m * quads) * 4, left = g.b.rows - n;
    if (m >= g.a.rows) return;
    const float* __restrict__ src = g.work + m * g.b.rows + n;
    f4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = 0; p < g.parts; ++p, src += (int64_t)g.a.rows * g.b.rows) {
        f4 v = {0.f, 0.f, 0.f, 0.f};
        if (left >= 4) __builtin_memcpy(&v, src, 16);
        else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < left) v[i] = src[i];
        }
        sum += v;
    }
    MatmulArgs whole = g;
    whole.parts = 1;
    put4(whole, 0, (int)m, n, sum);
}

Fp8Plan fp8_matmul_plan(int cus, int64_t m, int64_t n, int64_t k, int type)
{
    Fp8Plan p;
    p.tm = p.tn = 128;
    const int64_t tiles = std::max<int64_t>(1, ((m + p.tm - 1) / p.tm) * ((n + p.tn - 1) / p.tn)), blocks = (k + 127) / 128;
    const int64_t want = std::min<int64_t>(std::max<int64_t>(1, cus / tiles), std::max<int64_t>(1, blocks / 4));
    p.blocks_per_part = std::max<int64_t>(1, (blocks + want - 1) / want);
    p.parts = (int)std::max<int64_t>(1, (blocks + p.blocks_per_part - 1) / p.blocks_per_part);
    return p;
}

int64_t fp8_matmul_workspace(const Fp8Plan& p, int64_t m, int64_t n) { return p.parts > 1 ? p.parts * m * n * (int64_t)sizeof(float) : 0; }

template <int FA, int FB, int PER>
static hipError_t matmul_of(hipStream_t s, const Fp8Plan& p, const MatmulArgs& g)
{
    const dim3 grid((unsigned)((g.a.rows + p.tm - 1) / p.tm), (unsigned)((g.b.rows + p.tn - 1) / p.tn), (unsigned)p.parts);
    if (g.type == FOBQ_F32) hipLaunchKernelGGL((fp8_matmul_kernel<128, 128, 2, 2, FA, FB, PER, true>), grid, dim3(256), 0, s, g);
    else hipLaunchKernelGGL((fp8_matmul_kernel<128, 128, 2, 2, FA, FB, PER, false>), grid, dim3(256), 0, s, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    const int64_t items = (int64_t)g.a.rows * ((g.b.rows + 3) / 4);
    hipLaunchKernelGGL(fp8_matmul_join_kernel, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, s, g);
    return hipGetLastError();
}

template <int FA, int FB>
static hipError_t matmul_of(hipStream_t s, const Fp8Plan& p, const MatmulArgs& g)
{
    return g.b.per == 1 ? matmul_of<FA, FB, 1>(s, p, g) : matmul_of<FA, FB, 128>(s, p, g);
}

hipError_t launch_fp8_matmul(hipStream_t s, const Fp8Plan& p, const Fp8View& a, const Fp8View& b, void* y, int type, int64_t ldy, float* work)
{
    const MatmulArgs g{a, b, y, type, ldy, work, p.parts, (int)p.blocks_per_part};
    if (a.format == FOBQ_E4M3) return b.format == FOBQ_E4M3 ? matmul_of<0, 0>(s, p, g) : matmul_of<0, 1>(s, p, g);
    return b.format == FOBQ_E4M3 ? matmul_of<1, 0>(s, p, g) : matmul_of<1, 1>(s, p, g);
}

}  // namespace fobq
