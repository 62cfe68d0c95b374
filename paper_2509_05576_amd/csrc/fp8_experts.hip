// Products of each expert's rows with that expert's weights, matrices in 8-bit floating point with a scale for each block of 128 columns:
//   Y[p][n] = sum_kb sa[kb][a(p)] sb_e[kb][n / per] sum_{k in block kb} A[a(p)][k] B_e[n][k]      for the packed rows p of expert e
// Sums, matrix instructions and the places in LDS are those of a product of two matrices (fp8_matmul.hip).  What differs: where an expert's rows begin
// is known on the device only.  A launch has a workgroup for each tile that there can be at most; each finds the tiles of all experts in front of its own by one
// ascending sum over a wavefront, and those behind the last tile end.
#include "fp8_tile.h"

#include <algorithm>

namespace fobq {

// A workgroup's tile: `there` packed rows from `row` on, of expert `expert`, and B's rows from n0.  there 0: none.
struct ExpertTile { int expert, row, there, n0; };

// Tiles of TM rows and TN of B's.  Workgroups go to the 8 XCDs in turn, and each XCD has a run of tiles.  Within an expert up to 8 tiles of rows go
// along B's rows together, so that they share those in the XCD's L2.
__device__ __forceinline__ ExpertTile expert_tile(const ExpertView& g, int TM, int TN)
{
    const int lane = threadIdx.x & 63, per = (g.experts + 63) / 64;      // a lane has `per` neighbouring experts
    auto inside = [&](int v) { return min(max(v, 0), g.rows); };
    auto begin = [&](int e) { return inside(g.starts[e]); };
    auto count = [&](int e) { return max(inside(g.starts[e + 1]) - begin(e), 0); };
    int mine = 0;
    for (int i = 0; i < per; ++i) {
        const int e = lane * per + i;
        if (e < g.experts) mine += (count(e) + TM - 1) / TM;
    }
    int sum = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(sum, off);
        if (lane >= off) sum += v;
    }
    const int tiles_n = (g.b.rows + TN - 1) / TN;
    const int64_t tiles = (int64_t)__builtin_amdgcn_readlane(sum, 63) * tiles_n;
    const int xcd = blockIdx.x % 8, index = blockIdx.x / 8;
    if (index >= tiles / 8 + (xcd < tiles % 8)) return ExpertTile{0, 0, 0, 0};
    const int64_t at = tiles / 8 * xcd + min((int64_t)xcd, tiles % 8) + index;
    const int down = (int)(at / tiles_n);                    // tiles of rows in front
    const int owner = __popcll(__ballot(sum <= down));       // the lane whose experts have it
    if (owner > 63) return ExpertTile{0, 0, 0, 0};
    int before = __builtin_amdgcn_readlane(sum - mine, owner), expert = owner * per;
    for (int i = 0; i < per; ++i, ++expert) {
        if (expert >= g.experts) return ExpertTile{0, 0, 0, 0};
        const int n = (count(expert) + TM - 1) / TM;
        if (down < before + n) break;
        before += n;
    }
    if (expert >= owner * per + per) return ExpertTile{0, 0, 0, 0};      // (not with starts that ascend)
    const int rows = count(expert), tiles_m = (rows + TM - 1) / TM;
    const int in_expert = (int)(at - (int64_t)before * tiles_n);
    const int strip = in_expert / (8 * tiles_n), in_strip = in_expert - strip * 8 * tiles_n, high = min(8, tiles_m - 8 * strip);
    if (high <= 0) return ExpertTile{0, 0, 0, 0};
    const int m0 = (8 * strip + in_strip % high) * TM;
    return ExpertTile{expert, begin(expert) + m0, min(TM, rows - m0), in_strip / high * TN};
}

// The row of A that packed row p has, or -1.
__device__ __forceinline__ int row_of_a(const ExpertView& g, int p)
{
    if (!g.pairs) return p;
    const int pair = g.pairs[p];
    const unsigned row = (unsigned)pair / (unsigned)g.top;
    return pair >= 0 && row < (unsigned)g.a.rows ? (int)row : -1;
}

// four consecutive n of packed row p
__device__ __forceinline__ void put4(const ExpertView& g, int p, int n, f4 v)
{
    const int left = g.b.rows - n;
    auto out = [&](auto zero) {
        using T = decltype(zero);
        T* dst = static_cast<T*>(g.y) + (int64_t)p * g.ldy + n;
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

// 16 bytes a lane from its own address into LDS, lane after lane
__device__ __forceinline__ void copy16_from(const uint8_t* src, void* lds_base)
{
    __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)src, (void __attribute__((address_space(3)))*)lds_base, 16, 0, 0);
}

// TM x TN outputs by WM x WN wavefronts, the tiles of STAGES - 1 blocks under way.  FA, FB: the types of A and B; PER: rows of B to a scale.
template <int TM, int TN, int WM, int WN, int STAGES, int FA, int FB, int PER, bool EXACT>
__global__ __launch_bounds__(64 * WM * WN) void fp8_experts_kernel(ExpertView g)
{
    constexpr int WAVES = WM * WN, THREADS = 64 * WAVES, SM = TM / WM / 16, SN = TN / WN / 16;
    // per stage: rows of A, rows of B, and the scales of each
    constexpr int ROWS = TM + TN, STAGE = ROWS * 132;
    __shared__ __attribute__((aligned(16))) uint8_t sh[STAGES][STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, c = lane & 15;
    const int wm = wave / WN, wn = wave % WN;
    const int N = g.b.rows, K = g.a.cols, blocks = (K + 127) / 128;
    const ExpertTile tile = expert_tile(g, TM, TN);
    if (tile.there == 0) return;
    const int expert = __builtin_amdgcn_readfirstlane(tile.expert), p0 = __builtin_amdgcn_readfirstlane(tile.row);
    const int M = __builtin_amdgcn_readfirstlane(tile.there), n0 = __builtin_amdgcn_readfirstlane(tile.n0);
    const uint8_t* const b_values = g.b.values + expert * g.expert_values;
    const float* const b_scales = g.b.scales + expert * g.expert_scales;

    // A tile is copied 16 bytes a thread and piece, its rows in LDS one after another: a piece is THREADS / 8 rows below the one before.
    // Rows of A behind the tile's last are that one again, and not stored; rows of B behind its last read as zeros.
    constexpr int PA = TM * 8 / THREADS, PB = TN * 8 / THREADS, STEP = THREADS / 8;
    static_assert(TM % STEP == 0 && TN % STEP == 0 && STEP % 16 == 0, "pieces of whole rows, the same place in each");
    const int row = threadIdx.x >> 3, column = swizzle(row, threadIdx.x & 7) * 16;
    const uint8_t* a_row[PA];
#pragma unroll
    for (int i = 0; i < PA; ++i) a_row[i] = g.a.values + (int64_t)max(row_of_a(g, p0 + min(i * STEP + row, M - 1)), 0) * g.a.ld;
    const Run rb = run_of(b_values + n0 * g.b.ld, (N - n0) * g.b.ld);
    const unsigned ldb = (unsigned)g.b.ld, ob = row * ldb + column;
    auto fetch_values = [&](int stage, int kb) {
#pragma unroll
        for (int i = 0; i < PA; ++i) copy16_from(a_row[i] + column + kb * 128, &sh[stage][(i * THREADS + wave * 64) * 16]);
#pragma unroll
        for (int i = 0; i < PB; ++i) copy16(rb, ob + (i * STEP) * ldb + (unsigned)kb * 128, &sh[stage][TM * 128 + (i * THREADS + wave * 64) * 16]);
    };
    // A block's scales, one for each row of A and of B: 64 a wavefront.  (With fewer of them than wavefronts some are copied twice.)
    static_assert(ROWS / 64 == WAVES || WAVES % (ROWS / 64) == 0, "every wavefront copies scales once");
    const int piece = wave % (ROWS / 64);
    const bool of_a = piece < TM / 64;
    const int scale0 = of_a ? 0 : n0 / PER, scales_there = of_a ? g.a.rows : (N + PER - 1) / PER - scale0;
    const unsigned scale_at = of_a ? (unsigned)max(row_of_a(g, p0 + min(piece * 64 + lane, M - 1)), 0) : (n0 + piece * 64 - TM + lane) / PER - scale0;
    const float* const scale_of = (of_a ? g.a.scales : b_scales) + scale0;
    const int64_t scale_ld = of_a ? g.a.ld_scales : g.b.ld_scales;
    auto fetch_scales = [&](int stage, int kb) {
        copy4(run_of(scale_of + kb * scale_ld, (int64_t)scales_there * 4), scale_at * 4, &sh[stage][ROWS * 128 + piece * 256]);
    };
    constexpr int COPIES = PA + PB + 1;
    // the last block of columns where it is not whole: what is behind it counts as zero, whatever the rows hold there
    auto fetch_rest = [&](int stage, int kb) {
        const int k = kb * 128 + column, left = K - k;
        auto put = [&](const uint8_t* src, bool there, uint8_t* dst) {
            uint32_t w[4] = {0, 0, 0, 0};
            if (left > 0 && there) {
                __builtin_memcpy(w, __builtin_assume_aligned(src + k, 16), 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int have = left - 4 * j;
                    w[j] &= have >= 4 ? 0xffffffffu : have <= 0 ? 0u : (1u << (8 * have)) - 1;
                }
            }
            __builtin_memcpy(__builtin_assume_aligned(dst, 16), w, 16);
        };
#pragma unroll
        for (int i = 0; i < PA; ++i) put(a_row[i], true, &sh[stage][(i * THREADS + threadIdx.x) * 16]);
        for (int i = 0; i < PB; ++i) {
            const int at = n0 + i * STEP + row;
            put(b_values + at * g.b.ld, at < N, &sh[stage][TM * 128 + (i * THREADS + threadIdx.x) * 16]);
        }
    };
    const int place0 = swizzle(c, 2 * q) * 16, place1 = swizzle(c, 2 * q + 1) * 16;
    auto fragment = [&](int stage, int first_row) {
        const uint8_t* p = &sh[stage][(first_row + c) * 128];
        const i4 lo = *reinterpret_cast<const i4*>(p + place0), hi = *reinterpret_cast<const i4*>(p + place1);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f4 acc[SM][SN];
#pragma unroll
    for (int i = 0; i < SM; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    const int wm0 = wm * (TM / WM), wn0 = wn * (TN / WN);
    // Rows of A in groups of 16, one behind the other: while the matrix instructions of a group run, the sums of the one before are added
    // up and the next one's operand comes from LDS.
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
    const int whole = K / 128;                               // blocks that are whole
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k)
        if (k < whole) {
            fetch_values(k, k);
            fetch_scales(k, k);
        }
    int stage = 0;
    for (int kb = 0; kb < whole; ++kb) {
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
    if (whole < blocks) {
        wait_and_meet<0>();
        fetch_rest(0, whole);
        fetch_scales(0, whole);
        wait_and_meet<0>();
        multiply(0);
    }
#pragma unroll
    for (int i = 0; i < SM; ++i) {
        const int m = wm0 + 16 * i + c;
        if (m < M && row_of_a(g, p0 + m) >= 0)
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                const int n = n0 + wn0 + 16 * j + 4 * q;
                if (n < N) put4(g, p0 + m, n, acc[i][j]);
            }
    }
}

ExpertPlan expert_plan(int cus, int64_t rows, int experts, int64_t n, int64_t k, int type, int per)
{
    ExpertPlan p;
    p.tm = p.tn = 64;
    // Each expert with rows has at least one tile, and one more for every tm rows further.
    const int64_t with_rows = std::min<int64_t>(rows, experts);
    p.tiles = (with_rows + (rows - with_rows) / p.tm) * ((n + p.tn - 1) / p.tn);
    return p;
}

template <int FA, int FB, int PER>
static hipError_t experts_of(hipStream_t s, const ExpertPlan& p, const ExpertView& g)
{
    const dim3 grid((unsigned)p.tiles);
    if (g.type == FOBQ_F32) hipLaunchKernelGGL((fp8_experts_kernel<64, 64, 2, 2, 4, FA, FB, PER, true>), grid, dim3(256), 0, s, g);
    else hipLaunchKernelGGL((fp8_experts_kernel<64, 64, 2, 2, 4, FA, FB, PER, false>), grid, dim3(256), 0, s, g);
    return hipGetLastError();
}

template <int FA, int FB>
static hipError_t experts_of(hipStream_t s, const ExpertPlan& p, const ExpertView& g)
{
    return g.b.per == 1 ? experts_of<FA, FB, 1>(s, p, g) : experts_of<FA, FB, 128>(s, p, g);
}

hipError_t launch_expert_matmul(hipStream_t s, const ExpertPlan& p, const ExpertView& g)
{
    if (g.a.format == FOBQ_E4M3) return g.b.format == FOBQ_E4M3 ? experts_of<0, 0>(s, p, g) : experts_of<0, 1>(s, p, g);
    return g.b.format == FOBQ_E4M3 ? experts_of<1, 0>(s, p, g) : experts_of<1, 1>(s, p, g);
}

}  // namespace fobq
