// Product of two matrices in 8-bit floating point with a scale for each block of 128 columns:
//   Y[m][n] = sum_kb sa[kb][m] sb[kb][n / per] sum_{k in block kb} A[m][k] B[n][k]
// The outer sum is a multiply-add per value and block on the vector units, in fp32: acc += (sa sb) * part, or, with a scale per row of B, acc +=
// sa * (sb * part) (scales whose product or whose product with a part passes fp32 give what fp32 gives).  The inner one is
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
// Tiles of both matrices are copied straight into LDS, 128 bytes a row, the 16-byte pieces of row r at places p ^ ((r ^ r / 8 % 2) % 8):
// eight rows, and 16, that lanes read at once then lie in all banks (with r / 2 % 8 a read took four cycles more).  Which k's a lane holds does
// not matter, as both operands have the same.
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

// 16 or 4 bytes a lane from `offset` of a run of memory into LDS, lane after lane.  Behind the run's end nothing is read.
typedef __amdgpu_buffer_rsrc_t Run;
__device__ __forceinline__ Run run_of(const void* p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)min(bytes, (int64_t)0xffffffff), 0x00020000);
}
__device__ __forceinline__ void copy16(Run run, unsigned offset, void* lds_base)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(run, (void __attribute__((address_space(3)))*)lds_base, 16, (int)offset, 0, 0, 0);
}
__device__ __forceinline__ void copy4(Run run, unsigned offset, void* lds_base)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(run, (void __attribute__((address_space(3)))*)lds_base, 4, (int)offset, 0, 0, 0);
}

// the place of a row's 16-byte piece
__device__ __forceinline__ int swizzle(int row, int piece) { return piece ^ ((row ^ (row >> 3 & 1)) & 7); }

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

constexpr int FEW_WAVES = 8, FEW_ROWS = 16;      // wavefronts of a workgroup for few rows of A, and how many those are

// Waits until at most LEFT copies of this wavefront are under way, and for the whole workgroup to be there.  (A barrier of the language
// waits for all of them.)
template <int LEFT>
__device__ __forceinline__ void wait_and_meet()
{
    static_assert(LEFT < 64, "a count of six bits");
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// TM x TN outputs by WM x WN wavefronts, the tiles of STAGES - 1 blocks under way.  FA, FB: the types of A and B; PER: rows of B to a scale.
// (8192^3, a scale per 128 x 128, bf16 results: 487 to 495 us, 2.26 PFLOP/s, with the matrix units busy for 51 % of the cycles and the vector units,
// the sums' multiply-adds, for 48 % beside them, at a clock that power keeps near 2 GHz; a library's plain 8-bit product, without scales
// of blocks, takes 411.  4096^3: 66 us; with a scale per row of B, a multiplication more for each sum, 95; EXACT 148.)
template <int TM, int TN, int WM, int WN, int STAGES, int FA, int FB, int PER, bool EXACT>
__global__ __launch_bounds__(64 * WM * WN) void fp8_matmul_kernel(MatmulArgs g)
{
    constexpr int WAVES = WM * WN, THREADS = 64 * WAVES, SM = TM / WM / 16, SN = TN / WN / 16;
    // per stage: rows of A, rows of B, and the scales of each
    constexpr int ROWS = TM + TN, STAGE = ROWS * 132;
    __shared__ __attribute__((aligned(16))) uint8_t sh[STAGES][STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, c = lane & 15;
    const int wm = wave / WN, wn = wave % WN;
    const int M = g.a.rows, N = g.b.rows, K = g.a.cols, blocks = (K + 127) / 128;
    // Workgroups go to the 8 XCDs in turn.  Each XCD has a run of tiles, in strips of 4 tile rows, so that the ones it works on at a
    // time share rows of A and of B in its L2.
    const int tiles_m = (M + TM - 1) / TM, tiles_n = (N + TN - 1) / TN, tiles = tiles_m * tiles_n;
    const int xcd = blockIdx.x % 8, first = tiles / 8 * xcd + min(xcd, tiles % 8), at = first + (int)blockIdx.x / 8;
    const int strip = at / (4 * tiles_n), in_strip = at - strip * 4 * tiles_n, high = min(4, tiles_m - 4 * strip);
    const int m0 = (4 * strip + in_strip % high) * TM, n0 = in_strip / high * TN, part = blockIdx.y;
    const int kb0 = part * g.per_part, kb1 = min(blocks, kb0 + g.per_part);

    // A tile is copied 16 bytes a thread and piece, its rows in LDS one after another: a piece is THREADS / 8 rows below the one before.
    // Rows behind the last read as zeros.
    constexpr int PA = TM * 8 / THREADS, PB = TN * 8 / THREADS, STEP = THREADS / 8;
    static_assert(TM % STEP == 0 && TN % STEP == 0 && STEP % 16 == 0, "pieces of whole rows, the same place in each");
    const int row = threadIdx.x >> 3, column = swizzle(row, threadIdx.x & 7) * 16;
    const Run ra = run_of(g.a.values + m0 * g.a.ld, (M - m0) * g.a.ld), rb = run_of(g.b.values + n0 * g.b.ld, (N - n0) * g.b.ld);
    const unsigned lda = (unsigned)g.a.ld, ldb = (unsigned)g.b.ld, oa = row * lda + column, ob = row * ldb + column;
    auto fetch_values = [&](int stage, int kb) {
#pragma unroll
        for (int i = 0; i < PA; ++i) copy16(ra, oa + (i * STEP) * lda + (unsigned)kb * 128, &sh[stage][(i * THREADS + wave * 64) * 16]);
#pragma unroll
        for (int i = 0; i < PB; ++i) copy16(rb, ob + (i * STEP) * ldb + (unsigned)kb * 128, &sh[stage][TM * 128 + (i * THREADS + wave * 64) * 16]);
    };
    // A block's scales, one for each row of A and of B: 64 a wavefront.  (With fewer of them than wavefronts some are copied twice.)
    static_assert(ROWS / 64 == WAVES || WAVES % (ROWS / 64) == 0, "every wavefront copies scales once");
    const int piece = wave % (ROWS / 64);
    const bool of_a = piece < TM / 64;
    const int scale0 = of_a ? m0 : n0 / PER, scales_there = of_a ? M - m0 : (N + PER - 1) / PER - scale0;
    const unsigned scale_at = of_a ? piece * 64 + lane : (n0 + piece * 64 - TM + lane) / PER - scale0;
    const float* const scale_of = (of_a ? g.a.scales : g.b.scales) + scale0;
    const int64_t scale_ld = of_a ? g.a.ld_scales : g.b.ld_scales;
    auto fetch_scales = [&](int stage, int kb) {
        copy4(run_of(scale_of + kb * scale_ld, (int64_t)scales_there * 4), scale_at * 4, &sh[stage][ROWS * 128 + piece * 256]);
    };
    constexpr int COPIES = PA + PB + 1;
    // the last block of columns where it is not whole: what is behind it counts as zero, whatever the rows hold there
    auto fetch_rest = [&](int stage, int kb) {
        const int k = kb * 128 + column, left = K - k;
        auto put = [&](const Fp8View& x, int at, int rows, uint8_t* dst) {
            uint32_t w[4] = {0, 0, 0, 0};
            if (left > 0 && at < rows) {
                __builtin_memcpy(w, __builtin_assume_aligned(x.values + at * x.ld + k, 16), 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int have = left - 4 * j;
                    w[j] &= have >= 4 ? 0xffffffffu : have <= 0 ? 0u : (1u << (8 * have)) - 1;
                }
            }
            __builtin_memcpy(__builtin_assume_aligned(dst, 16), w, 16);
        };
        for (int i = 0; i < PA; ++i) put(g.a, m0 + i * STEP + row, M, &sh[stage][(i * THREADS + threadIdx.x) * 16]);
        for (int i = 0; i < PB; ++i) put(g.b, n0 + i * STEP + row, N, &sh[stage][TM * 128 + (i * THREADS + threadIdx.x) * 16]);
    };
    const int p0 = swizzle(c, 2 * q) * 16, p1 = swizzle(c, 2 * q + 1) * 16;
    auto fragment = [&](int stage, int first_row) {
        const uint8_t* p = &sh[stage][(first_row + c) * 128];
        const i4 lo = *reinterpret_cast<const i4*>(p + p0), hi = *reinterpret_cast<const i4*>(p + p1);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f4 acc[SM][SN];
#pragma unroll
    for (int i = 0; i < SM; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    const int wm0 = wm * (TM / WM), wn0 = wn * (TN / WN);
    // Rows of A in groups of 16, one behind the other: while the matrix instructions of a group run, the sums of the one before are added
    // up and the next one's operand comes from LDS.  The order is kept; the compiler's own has every instruction wait for the one before.
    auto multiply = [&](int stage) {
        using BF = decltype(operand<EXACT, FB>(i8v()));
        using AF = decltype(operand<EXACT, FA>(i8v()));
        const float* scales = reinterpret_cast<const float*>(&sh[stage][ROWS * 128]);
        BF bf[SN];
        AF af[2];
        f4 p[2][SN], sb[PER == 1 ? SN : 1];
        float sa[SM];
        af[0] = operand<EXACT, FA>(fragment(stage, wm0));
#pragma unroll
        for (int j = 0; j < SN; ++j) bf[j] = operand<EXACT, FB>(fragment(stage, TM + wn0 + 16 * j));
#pragma unroll
        for (int i = 0; i < SM; ++i) sa[i] = scales[wm0 + 16 * i + c];
        if constexpr (PER == 1) {
#pragma unroll
            for (int j = 0; j < SN; ++j) sb[j] = *reinterpret_cast<const f4*>(&scales[TM + wn0 + 16 * j + 4 * q]);
        } else {
            sb[0][0] = scales[TM + wn0];
        }
#pragma unroll
        for (int i = 0; i <= SM; ++i) {
            if (i + 1 < SM) af[(i + 1) & 1] = operand<EXACT, FA>(fragment(stage, wm0 + 16 * (i + 1)));
            const float s = i == 0 ? 0.f : PER == 1 ? sa[i - 1] : sa[i - 1] * sb[0][0];
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                if (i < SM) p[i & 1][j] = mfma_block<FB, FA>(bf[j], af[i & 1]);
                if (i > 0) {
                    f4& d = acc[i - 1][j];
                    const f4 x = p[(i - 1) & 1][j];
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] = fmaf(PER == 1 ? x[e] * sb[PER == 1 ? j : 0][e] : x[e], s, d[e]);
                }
                if (!EXACT) __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    const int whole = min(kb1, K / 128);                     // blocks of this part that are whole
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k)
        if (kb0 + k < whole) {
            fetch_values(k, kb0 + k);
            fetch_scales(k, kb0 + k);
        }
    int stage = 0;
    for (int kb = kb0; kb < whole; ++kb) {
        if (kb + STAGES - 2 < whole) wait_and_meet<(STAGES - 2) * COPIES>();
        else wait_and_meet<0>();
        // everybody is done with the block before: its stage is free
        if (kb + STAGES - 1 < whole) {
            const int free = stage == 0 ? STAGES - 1 : stage - 1;
            fetch_values(free, kb + STAGES - 1);
            fetch_scales(free, kb + STAGES - 1);
        }
        multiply(stage);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    if (whole < kb1) {
        wait_and_meet<0>();
        fetch_rest(0, whole);
        fetch_scales(0, whole);
        wait_and_meet<0>();
        multiply(0);
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

// Up to 16 rows of A: the weights are read once, straight into the registers of the wavefront that multiplies them, 128 bytes of 16 rows in
// two loads.  A workgroup has 16 rows of B; its wavefronts deal the blocks among them, four at a time (8 KiB of weights in flight each), and
// add up in LDS, in their order.  On fp16 values throughout: conversions are hidden behind memory.  (n = k = 8192: 1 row 14.0 us, 4.8 TB/s, as
// a large copy; 16 rows with a scale per row of B 18 us.)
template <int FA, int FB, int PER>
__global__ __launch_bounds__(64 * FEW_WAVES) void fp8_matmul_few_kernel(MatmulArgs g)
{
    constexpr int AT_ONCE = 4;
    __shared__ f4 sum[FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
    const int M = g.a.rows, N = g.b.rows, K = g.a.cols, blocks = (K + 127) / 128;
    const int n0 = blockIdx.x * 16;
    const uint8_t* __restrict__ brow = g.b.values + (int64_t)min(n0 + c, N - 1) * g.b.ld + 32 * q;
    const uint8_t* __restrict__ arow = g.a.values + (int64_t)min(c, M - 1) * g.a.ld + 32 * q;
    f4 acc = {0.f, 0.f, 0.f, 0.f};

    auto load = [&](const uint8_t* __restrict__ row, int kb) {
        i4 lo, hi;
        const int k = kb * 128 + 32 * q;
        if (kb * 128 + 128 <= K) {
            lo = *reinterpret_cast<const i4*>(row + (int64_t)kb * 128);
            hi = *reinterpret_cast<const i4*>(row + (int64_t)kb * 128 + 16);
        } else {
            // the last block, which is not whole, and those behind it: nothing is read there
            auto piece = [&](int at) {
                i4 w = {0, 0, 0, 0};
                if (at < K) {
                    w = *reinterpret_cast<const i4*>(row + (at - 32 * q));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int have = K - at - 4 * j;
                        w[j] &= have >= 4 ? -1 : have <= 0 ? 0 : (1 << (8 * have)) - 1;
                    }
                }
                return w;
            };
            lo = piece(k);
            hi = piece(k + 16);
        }
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    for (int kb0 = wave * AT_ONCE; kb0 < blocks; kb0 += FEW_WAVES * AT_ONCE) {
        i8v b[AT_ONCE], a[AT_ONCE];
        float sa[AT_ONCE], sb[AT_ONCE][PER == 1 ? 4 : 1];
#pragma unroll
        for (int x = 0; x < AT_ONCE; ++x) {
            b[x] = load(brow, kb0 + x);
            const int kb = min(kb0 + x, blocks - 1);
            a[x] = load(arow, kb0 + x);
            sa[x] = g.a.scales[kb * g.a.ld_scales + min(c, M - 1)];
            if constexpr (PER == 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sb[x][e] = g.b.scales[kb * g.b.ld_scales + min(n0 + 4 * q + e, N - 1)];
            } else {
                sb[x][0] = g.b.scales[kb * g.b.ld_scales + n0 / 128];
            }
        }
#pragma unroll
        for (int x = 0; x < AT_ONCE; ++x) {
            if (kb0 + x >= blocks) break;
            const f4 p = mfma_block<FB, FA>(as_fp16<FB>(b[x]), as_fp16<FA>(a[x]));
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e] * sb[x][PER == 1 ? e : 0], sa[x], acc[e]);
        }
    }
    sum[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
        f4 v = sum[0][lane];
#pragma unroll
        for (int k = 1; k < FEW_WAVES; ++k) v += sum[k][lane];
        const int n = n0 + 4 * q;
        if (c < M && n < N) put4(g, 0, c, n, v);
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

// The measurements behind the rules (bf16 results, a scale per 128 x 128, us; n = k = 8192 where one number is given):
//   up to 16 rows         one kernel for few rows: 13.2 with 1 row; with 17 and 32 rows 21 and 26 against 16 and 17 in tiles of 64
//   64, 128 or 256        1024 rows 136, 89, 104; 2048 rows 262, 169, 127; 300 x 4608 x 2048 10.8, 16.8, 33; 2000^3 26, 21, 35;
//                         4096^3 134, 91, 65; 1500 x 6000 x 3000 65, 55, 50.  A compute unit has one workgroup of the largest tiles at a
//                         time or two of the others, and the larger of two takes less per value, 1 : 1.4
//   parts of the sum      64 rows, 128 tiles of 64 blocks: 25 in one part, 19 in two and in four; 128 rows, 256 tiles: 26 and 27;
//                         500 x 1000 x 2304, 18 blocks: 10 and 14 (the second launch takes 4.5)
Fp8Plan fp8_matmul_plan(int cus, int64_t m, int64_t n, int64_t k, int type, int per)
{
    Fp8Plan p;
    const int64_t blocks = (k + 127) / 128;
    auto tiles = [&](int64_t t) { return ((m + t - 1) / t) * ((n + t - 1) / t); };
    auto rounds = [&](int64_t t, int64_t at_once) { return (tiles(t) + at_once - 1) / at_once; };
    int64_t want = 1;
    if (m <= FEW_ROWS) {
        p.tm = p.tn = FEW_ROWS;
    } else if (type != FOBQ_F32 && per == 128 && 10 * rounds(256, cus) <= 7 * rounds(128, 2 * cus)) {
        p.tm = p.tn = 256;              // (results in 32 bits, or a scale per row of B, take more registers than there are)
    } else if (tiles(128) >= cus) {
        p.tm = p.tn = 128;
    } else {
        p.tm = p.tn = 64;
        if (tiles(64) < cus) want = std::max<int64_t>(1, std::min(2 * cus / std::max<int64_t>(1, tiles(64)), blocks / 16));
    }
    p.blocks_per_part = std::max<int64_t>(1, (blocks + want - 1) / want);
    p.parts = (int)std::max<int64_t>(1, (blocks + p.blocks_per_part - 1) / p.blocks_per_part);
    return p;
}

int64_t fp8_matmul_workspace(const Fp8Plan& p, int64_t m, int64_t n) { return p.parts > 1 ? p.parts * m * n * (int64_t)sizeof(float) : 0; }

template <int FA, int FB, int PER>
static hipError_t matmul_of(hipStream_t s, const Fp8Plan& p, const MatmulArgs& g)
{
    const dim3 grid((unsigned)(((g.a.rows + p.tm - 1) / p.tm) * ((g.b.rows + p.tn - 1) / p.tn)), (unsigned)p.parts);
    if (p.tm == FEW_ROWS) {
        hipLaunchKernelGGL((fp8_matmul_few_kernel<FA, FB, PER>), dim3((unsigned)((g.b.rows + 15) / 16)), dim3(64 * FEW_WAVES), 0, s, g);
        return hipGetLastError();
    }
    const bool exact = g.type == FOBQ_F32;
    if (p.tm == 256) {
        if constexpr (PER == 128) hipLaunchKernelGGL((fp8_matmul_kernel<256, 256, 2, 4, 2, FA, FB, PER, false>), grid, dim3(512), 0, s, g);
    } else if (p.tm == 128) {
        if (exact) hipLaunchKernelGGL((fp8_matmul_kernel<128, 128, 2, 2, 2, FA, FB, PER, true>), grid, dim3(256), 0, s, g);
        else hipLaunchKernelGGL((fp8_matmul_kernel<128, 128, 2, 2, 2, FA, FB, PER, false>), grid, dim3(256), 0, s, g);
    } else {
        if (exact) hipLaunchKernelGGL((fp8_matmul_kernel<64, 64, 2, 2, 4, FA, FB, PER, true>), grid, dim3(256), 0, s, g);
        else hipLaunchKernelGGL((fp8_matmul_kernel<64, 64, 2, 2, 4, FA, FB, PER, false>), grid, dim3(256), 0, s, g);
    }
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
