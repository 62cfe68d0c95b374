// Products of each expert's rows with that expert's weights, matrices in 8-bit floating point with a scale for each block of 128 columns:
//   Y[p][n] = sum_kb sa[kb][a(p)] sb_e[kb][n / per] sum_{k in block kb} A[a(p)][k] B_e[n][k]      for the packed rows p of expert e
// Sums, matrix instructions and the places in LDS are those of a product of two matrices (fp8_matmul.hip).  What differs: where an expert's rows begin
// is known on the device only.  A launch has a workgroup for each tile that there can be at most; each finds the tiles of all experts in front of its own by one
// ascending sum over a wavefront, and those behind the last tile end.
#include "fp8_tile.h"

#include <algorithm>
#include <type_traits>

namespace fobq {

// A workgroup's tile: `there` packed rows from `row` on, of expert `expert`, and B's rows from n0.  there 0: none.
struct ExpertTile { int expert, row, there, n0; };

// the sum of x over the lanes up to this one
__device__ __forceinline__ int sum_up_to(int x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(x, off);
        if (lane >= off) x += v;
    }
    return x;
}

// Tiles of TM rows and TN of B's.  Workgroups go to the 8 XCDs in turn, and each XCD has a run of tiles.  Within an expert up to 8 tiles of rows go
// along B's rows together, so that they share those in the XCD's L2.  A lane has `per` neighbouring experts: one look at all starts, and one at the
// starts of the lane that has the tile, if there are more than 64.
template <int TM, int TN>
__device__ __forceinline__ ExpertTile expert_tile(const ExpertView& g)
{
    const int lane = threadIdx.x & 63, per = (g.experts + 63) / 64;
    const ExpertTile none{0, 0, 0, 0};
    auto inside = [&](int v) { return min(max(v, 0), g.rows); };
    int begin = 0, rows = 0, tiles = 0;                      // of the lane's last expert; of all of the lane's
    auto look = [&](int e) {
        if (e >= g.experts) return;
        begin = inside(g.starts[e]);
        rows = max(inside(g.starts[e + 1]) - begin, 0);
        tiles += (rows + TM - 1) / TM;
    };
    for (int i = 0; i < per; ++i) look(lane * per + i);
    tiles = min(tiles, (1 << 25) - 1);                       // (fewer, with starts that ascend)
    int sum = sum_up_to(tiles);
    const int tiles_n = (g.b.rows + TN - 1) / TN;
    const unsigned all = (unsigned)min((int64_t)__builtin_amdgcn_readlane(sum, 63) * tiles_n, (int64_t)gridDim.x);
    const unsigned xcd = blockIdx.x % 8, index = blockIdx.x / 8;
    if (index >= all / 8 + (xcd < all % 8)) return none;
    const unsigned at = all / 8 * xcd + min(xcd, all % 8) + index;
    const int down = at / (unsigned)tiles_n;                 // tiles of rows in front
    int owner = __popcll(__ballot(sum <= down)), first = 0;
    if (owner > 63) return none;
    int before = __builtin_amdgcn_readlane(sum - tiles, owner);
    if (per > 1) {
        first = owner * per;
        tiles = 0;
        rows = 0;
        if (lane < per) look(first + lane);
        sum = sum_up_to(tiles) + before;
        owner = __popcll(__ballot(sum <= down));
        if (owner > 63) return none;
        before = __builtin_amdgcn_readlane(sum - tiles, owner);
    }
    begin = __builtin_amdgcn_readlane(begin, owner);
    rows = __builtin_amdgcn_readlane(rows, owner);
    const unsigned tiles_m = (rows + TM - 1) / TM, in_expert = at - (unsigned)before * (unsigned)tiles_n, strip = in_expert / (8u * tiles_n);
    const unsigned in_strip = in_expert - strip * 8 * tiles_n;
    if (8 * strip >= tiles_m) return none;
    const unsigned high = min(8u, tiles_m - 8 * strip), over = in_strip / high;
    const int m0 = (8 * strip + in_strip - over * high) * TM;
    return ExpertTile{first + owner, begin + m0, min(TM, rows - m0), (int)over * TN};
}

// The row of A that packed row p has, or -1.
__device__ __forceinline__ int row_of_a(const ExpertView& g, int p)
{
    if (!g.pairs) return p;
    const int pair = g.pairs[p];
    const unsigned row = (unsigned)pair / (unsigned)g.top;
    return pair >= 0 && row < (unsigned)g.a.rows ? (int)row : -1;
}

// N consecutive results from n on, as many of them as B has rows
template <int N, class T>
__device__ __forceinline__ void put(T* __restrict__ dst, int left, const T* t)
{
    if (left >= N) __builtin_memcpy(dst, t, N * sizeof(T));
    else {
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (i < left) dst[i] = t[i];
    }
}

// Two neighbouring tiles' results of 16 bits: a lane has four of each, at 4 q of 16, and gets eight of one of them, so that a row's 32 are stored in
// pieces of 16 bytes.  (lane / 16 = q odd: of the second; q >= 2: the upper eight.)
template <class T>
__device__ __forceinline__ void put_pair(T* __restrict__ row, int n, int N, f4 x, f4 y)
{
    typedef T two __attribute__((ext_vector_type(2)));
    auto pack = [](float a, float b) { return __builtin_bit_cast(uint32_t, two{(T)a, (T)b}); };
    const auto low = __builtin_amdgcn_permlane16_swap(pack(x[0], x[1]), pack(y[0], y[1]), false, false);
    const auto high = __builtin_amdgcn_permlane16_swap(pack(x[2], x[3]), pack(y[2], y[3]), false, false);
    const uint32_t w[4] = {low[0], high[0], low[1], high[1]};
    T t[8];
    __builtin_memcpy(t, w, sizeof t);
    if (row && n < N) put<8>(row + n, N - n, t);
}

// 16 bytes a lane from its own address into LDS, lane after lane
__device__ __forceinline__ void copy16_from(const uint8_t* src, void* lds_base)
{
    __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)src, (void __attribute__((address_space(3)))*)lds_base, 16, 0, 0);
}

// TM x TN outputs by WM x WN wavefronts, the tiles of STAGES - 1 blocks under way.  FA, FB: the types of A and B; PER: rows of B to a scale.
// (32768 rows in 64 experts of 4096 x 2048, bf16, a scale per 128 x 128: 376 to 390 us, 1.41 to 1.46 PFLOP/s, in tiles of 256 x 256; with 512 packed rows in each expert 316, as one
// product of as many rows in whole tiles takes 299.  A tile's 16 blocks take 32 us, its start and end 6, of which the stores 4.7; a block's products alone take
// 1.47, its copies alone 1.71: LDS has both.  256 rows in 128 experts of 2048 x 2048: 80 us, 5.4 TB/s.)
// With PARTS above 1 as many such sets of wavefronts deal the blocks of columns among them, and add up in LDS, in their order.
template <int TM, int TN, int WM, int WN, int STAGES, int PARTS, int FA, int FB, int PER, bool EXACT>
__global__ __launch_bounds__(64 * WM * WN * PARTS) void fp8_experts_kernel(ExpertView g)
{
    constexpr int WAVES = WM * WN, THREADS = 64 * WAVES, SM = TM / WM / 16, SN = TN / WN / 16;
    // per stage: rows of A, rows of B, and the scales of each
    constexpr int ROWS = TM + TN, STAGE = ROWS * 132;
    __shared__ __attribute__((aligned(16))) uint8_t all[PARTS][STAGES][STAGE];
    const int tid = threadIdx.x % THREADS, lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint8_t(*const sh)[STAGE] = all[part];
    const int q = lane >> 4, c = lane & 15;
    const int wm = wave / WN, wn = wave % WN;
    const int N = g.b.rows, K = g.a.cols, blocks = (K + 127) / 128;
    const ExpertTile tile = expert_tile<TM, TN>(g);
    if (tile.there == 0) return;
    const int expert = __builtin_amdgcn_readfirstlane(tile.expert), p0 = __builtin_amdgcn_readfirstlane(tile.row);
    const int M = __builtin_amdgcn_readfirstlane(tile.there), n0 = __builtin_amdgcn_readfirstlane(tile.n0);
    const uint8_t* const b_values = g.b.values + expert * g.expert_values;
    const float* const b_scales = g.b.scales + expert * g.expert_scales;

    // A tile is copied 16 bytes a thread and piece, its rows in LDS one after another: a piece is THREADS / 8 rows below the one before.
    // Rows of A behind the tile's last are that one again, and not stored; rows of B behind its last read as zeros.
    // The copies of the block that is fetched stand between the products of the one that is multiplied, a few to each of the first 1 / SPREAD of its groups: all in front of
    // them, the first operands wait until the addresses of all are through.  With two stages they have to be under way by the middle, or the next block waits
    // for them.  (Both in turn, four times: 32768 rows in 64 experts of 4096 x 2048 391 -> 386 us, no more than a run differs from the next; with a scale per row, 128 x 256, 477 -> 454;
    // 16384 rows in 64 of 1024 x 2048 71.5 -> 65.8; 1400 rows in 8 of 1024 x 4096 20.0 -> 18.7.  On fp16 values, whose order is the compiler's, 427 -> 560: not there.)
    constexpr int SPREAD = PARTS > 1 || EXACT ? 0 : STAGES == 2 ? 2 : 1;
    constexpr int PA = TM * 8 / THREADS, PB = TN * 8 / THREADS, STEP = THREADS / 8;
    static_assert(TM % STEP == 0 && TN % STEP == 0 && STEP % 16 == 0, "pieces of whole rows, the same place in each");
    const int row = tid >> 3, column = swizzle(row, tid & 7) * 16;
    int at_a[PA];
#pragma unroll
    for (int i = 0; i < PA; ++i) at_a[i] = row_of_a(g, p0 + min(i * STEP + row, M - 1));
    const Run rb = run_of(b_values + n0 * g.b.ld, (N - n0) * g.b.ld);
    const unsigned ldb = (unsigned)g.b.ld, ob = row * ldb + column;
    auto copy_b = [&](int stage, int kb, int i) __attribute__((always_inline)) {
        copy16(rb, ob + (i * STEP) * ldb + (unsigned)kb * 128, &sh[stage][TM * 128 + (i * THREADS + wave * 64) * 16]);
    };
    auto fetch_b = [&](int stage, int kb) {
#pragma unroll
        for (int i = 0; i < PB; ++i) copy_b(stage, kb, i);
    };
    // A block's scales, one for each row of A and of B: 64 a wavefront.  (With fewer of them than wavefronts some are copied twice.)
    static_assert(ROWS / 64 <= WAVES, "every wavefront copies scales once");
    const int piece = wave % (ROWS / 64);
    const bool of_a = piece < TM / 64;
    const int scale0 = of_a ? 0 : n0 / PER, scales_there = of_a ? g.a.rows : (N + PER - 1) / PER - scale0;
    const unsigned scale_at = of_a ? (unsigned)max(row_of_a(g, p0 + min(piece * 64 + lane, M - 1)), 0) : (n0 + piece * 64 - TM + lane) / PER - scale0;
    const float* const scale_of = (of_a ? g.a.scales : b_scales) + scale0;
    const int64_t scale_ld = of_a ? g.a.ld_scales : g.b.ld_scales;
    // (the tile's own part of B needs no rows of A to be known)
    const int whole = K / 128, mine = (whole - part + PARTS - 1) / PARTS, steps = (whole + PARTS - 1) / PARTS;     // blocks that are whole, and the part's
    auto block = [&](int i) { return part + PARTS * i; };
    if (mine > 0) fetch_b(0, block(0));
    const uint8_t* a_row[PA];
#pragma unroll
    for (int i = 0; i < PA; ++i) a_row[i] = g.a.values + (int64_t)max(at_a[i], 0) * g.a.ld;
    auto copy_a = [&](int stage, int kb, int i) __attribute__((always_inline)) {
        copy16_from(a_row[i] + column + kb * 128, &sh[stage][(i * THREADS + wave * 64) * 16]);
    };
    auto fetch_a = [&](int stage, int kb, auto pieces) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < decltype(pieces)::value; ++i) copy_a(stage, kb, i);
    };
    auto fetch_scales = [&](int stage, int kb) {
        copy4(run_of(scale_of + kb * scale_ld, (int64_t)scales_there * 4), scale_at * 4, &sh[stage][ROWS * 128 + piece * 256]);
    };
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
        for (int i = 0; i < PA; ++i) put(a_row[i], true, &sh[stage][(i * THREADS + tid) * 16]);
        for (int i = 0; i < PB; ++i) {
            const int at = n0 + i * STEP + row;
            put(b_values + at * g.b.ld, at < N, &sh[stage][TM * 128 + (i * THREADS + tid) * 16]);
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

    const int wn0 = wn * (TN / WN);
    // A wavefront's groups of 16 rows of A: every WM-th of the tile's, those of them that have rows.
    auto group = [&](int i) { return 16 * (WM * i + wm); };
    unsigned stored = 0;                                     // bit i: the lane's row of group i is written
#pragma unroll
    for (int i = 0; i < SM; ++i) stored |= (unsigned)(group(i) + c < M && row_of_a(g, p0 + min(group(i) + c, M - 1)) >= 0) << i;
    // One group behind the other: while the matrix instructions of a group run, the sums of the one before are added up and the next one's operand
    // comes from LDS; between(i) follows the first of them.  The order is kept; the compiler's own has every instruction wait for the one before.
    auto multiply = [&](int stage, auto groups, auto between) __attribute__((always_inline)) {
        constexpr int G = decltype(groups)::value;
        using BF = decltype(operand<EXACT, FB>(i8v()));
        using AF = decltype(operand<EXACT, FA>(i8v()));
        const float* scales = reinterpret_cast<const float*>(&sh[stage][ROWS * 128]);
        BF bf[SN];
        AF af[2];
        f4 p[2][SN], sb[PER == 1 ? SN : 1];
        float sa[G];
        af[0] = operand<EXACT, FA>(fragment(stage, group(0)));
#pragma unroll
        for (int j = 0; j < SN; ++j) bf[j] = operand<EXACT, FB>(fragment(stage, TM + wn0 + 16 * j));
#pragma unroll
        for (int i = 0; i < G; ++i) sa[i] = scales[group(i) + c];
        if constexpr (PER == 1) {
#pragma unroll
            for (int j = 0; j < SN; ++j) sb[j] = *reinterpret_cast<const f4*>(&scales[TM + wn0 + 16 * j + 4 * q]);
        } else {
            sb[0][0] = scales[TM + wn0];
        }
#pragma unroll
        for (int i = 0; i <= G; ++i) {
            if (i + 1 < G) af[(i + 1) & 1] = operand<EXACT, FA>(fragment(stage, group(i + 1)));
            const float s = i == 0 ? 0.f : PER == 1 ? sa[i - 1] : sa[i - 1] * sb[0][0];
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                if (i < G) p[i & 1][j] = mfma_block<FB, FA>(bf[j], af[i & 1]);
                if (i > 0) {
                    f4& d = acc[i - 1][j];
                    const f4 x = p[(i - 1) & 1][j];
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] = fmaf(PER == 1 ? x[e] * sb[PER == 1 ? j : 0][e] : x[e], s, d[e]);
                }
                if (!EXACT) __builtin_amdgcn_sched_barrier(0);
                if (j == 0) between(i);
            }
        }
    };
    // By groups of a wavefront: no rows of A behind them are copied either.
    auto product = [&](auto groups) __attribute__((always_inline)) {
        constexpr int USED = (decltype(groups)::value * 16 * WM + STEP - 1) / STEP, COPIES = USED + PB + 1;
        constexpr auto pieces = std::integral_constant<int, USED>();
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k)
            if (k < mine) {
                if (k > 0) fetch_b(k, block(k));
                fetch_a(k, block(k), pieces);
                fetch_scales(k, block(k));
            }
        auto nothing = [](int) __attribute__((always_inline)) {};
        int stage = 0, i = 0;
        if constexpr (SPREAD > 0) {
            constexpr int OVER = (decltype(groups)::value + SPREAD - 1) / SPREAD;
            for (; i + STAGES - 1 < steps; ++i) {
                wait_and_meet<(STAGES - 2) * COPIES>();
                // everybody is done with the block before: its stage is free
                const int free = stage == 0 ? STAGES - 1 : stage - 1, next = i + STAGES - 1;
                multiply(stage, groups, [&](int at) __attribute__((always_inline)) {
#pragma unroll
                    for (int k = 0; k < COPIES; ++k)
                        if (k * OVER / COPIES == at) {
                            if (k < PB) copy_b(free, next, k);
                            else if (k < PB + USED) copy_a(free, next, k - PB);
                            else fetch_scales(free, next);
                        }
                });
                stage = stage == STAGES - 1 ? 0 : stage + 1;
            }
        }
        for (; i < steps; ++i) {
            if (i + STAGES - 2 < mine) wait_and_meet<(STAGES - 2) * COPIES>();
            else wait_and_meet<0>();
            if (SPREAD == 0 && i + STAGES - 1 < mine) {
                const int free = stage == 0 ? STAGES - 1 : stage - 1;
                fetch_b(free, block(i + STAGES - 1));
                fetch_a(free, block(i + STAGES - 1), pieces);
                fetch_scales(free, block(i + STAGES - 1));
            }
            if (PARTS == 1 || i < mine) multiply(stage, groups, nothing);
            stage = stage == STAGES - 1 ? 0 : stage + 1;
        }
        if (whole < blocks) {
            wait_and_meet<0>();
            if (part == 0) {
                fetch_rest(0, whole);
                fetch_scales(0, whole);
            }
            wait_and_meet<0>();
            if (part == 0) multiply(0, groups, nothing);
        }
    };
    // A tile with few rows takes less: by quarters (the whole workgroup goes the same way).
    if constexpr (SM % 4 == 0 && !EXACT) {
        if (M <= TM / 4) product(std::integral_constant<int, SM / 4>());
        else if (M <= TM / 2) product(std::integral_constant<int, SM / 2>());
        else if (M <= TM / 4 * 3) product(std::integral_constant<int, SM / 4 * 3>());
        else product(std::integral_constant<int, SM>());
    } else {
        if (SM >= 2 && M <= TM / 2) product(std::integral_constant<int, (SM + 1) / 2>());
        else product(std::integral_constant<int, SM>());
    }

    if constexpr (PARTS > 1) {
        static_assert((PARTS - 1) * SM * SN * THREADS * 16 <= sizeof all, "room for the sums");
        f4* const sums = reinterpret_cast<f4*>(&all[0][0][0]);
        wait_and_meet<0>();
        if (part > 0) {
#pragma unroll
            for (int i = 0; i < SM * SN; ++i) sums[((part - 1) * SM * SN + i) * THREADS + tid] = acc[i / SN][i % SN];
        }
        wait_and_meet<0>();
        if (part > 0) return;
#pragma unroll
        for (int k = 0; k < (PARTS - 1) * SM * SN; ++k) acc[k / SN % SM][k % SN] += sums[k * THREADS + tid];
    }
    // four consecutive n of a lane's row of each group
#pragma unroll
    for (int i = 0; i < SM; ++i) {
        const bool there = (stored >> i & 1) != 0;
        if (16 * (WM * i + wm) >= M) continue;
        const int64_t p = p0 + group(i) + c;
        auto sixteen = [&](auto zero) {
            using T = decltype(zero);
            T* dst = there ? static_cast<T*>(g.y) + p * g.ldy : nullptr;
#pragma unroll
            for (int j = 0; j < SN; j += 2) put_pair(dst, n0 + wn0 + 16 * (j + (q & 1)) + 8 * (q >> 1), N, acc[i][j], acc[i][j + 1]);
        };
        if constexpr (EXACT) {
            if (there)
#pragma unroll
                for (int j = 0; j < SN; ++j) {
                    const int n = n0 + wn0 + 16 * j + 4 * q;
                    const float t[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    if (n < N) put<4>(static_cast<float*>(g.y) + p * g.ldy + n, N - n, t);
                }
        } else {
            if (g.type == FOBQ_BF16) sixteen((bf16_t)0.f);
            else sixteen((f16_t)0.f);
        }
    }
}

// Up to 16 rows of an expert at a time, straight from memory into the registers of the wavefronts that multiply them, on fp16 values: for calls
// whose weights are all there is to read.  A workgroup has 16 rows of B; its wavefronts deal the blocks among them, two at a time, and add up
// in LDS, in their order.
constexpr int FEW_WAVES = 8;
template <int FA, int FB, int PER>
__global__ __launch_bounds__(64 * FEW_WAVES) void fp8_experts_few_kernel(ExpertView g)
{
    constexpr int AT_ONCE = 2;
    __shared__ f4 sum[FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
    const ExpertTile tile = expert_tile<16, 16>(g);
    if (tile.there == 0) return;
    const int expert = __builtin_amdgcn_readfirstlane(tile.expert), p0 = __builtin_amdgcn_readfirstlane(tile.row);
    const int M = __builtin_amdgcn_readfirstlane(tile.there), n0 = __builtin_amdgcn_readfirstlane(tile.n0);
    const int N = g.b.rows, K = g.a.cols, blocks = (K + 127) / 128;
    const int at_a = row_of_a(g, p0 + min(c, M - 1)), row_a = max(at_a, 0);
    const float* const b_scales = g.b.scales + expert * g.expert_scales;
    const uint8_t* __restrict__ brow = g.b.values + expert * g.expert_values + (int64_t)min(n0 + c, N - 1) * g.b.ld + 32 * q;
    const uint8_t* __restrict__ arow = g.a.values + (int64_t)row_a * g.a.ld + 32 * q;
    f4 acc = {0.f, 0.f, 0.f, 0.f};

    auto load = [&](const uint8_t* __restrict__ row, int kb) {
        i4 lo, hi;
        if (kb * 128 + 128 <= K) {
            lo = *reinterpret_cast<const i4*>(row + (int64_t)kb * 128);
            hi = *reinterpret_cast<const i4*>(row + (int64_t)kb * 128 + 16);
        } else {
            // the last block, which is not whole, and those behind it: nothing is read there
            const int k = kb * 128 + 32 * q;
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
            sa[x] = g.a.scales[kb * g.a.ld_scales + row_a];
            if constexpr (PER == 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sb[x][e] = b_scales[kb * g.b.ld_scales + min(n0 + 4 * q + e, N - 1)];
            } else {
                sb[x][0] = b_scales[kb * g.b.ld_scales + n0 / 128];
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
    if (wave != 0) return;
    f4 v = sum[0][lane];
#pragma unroll
    for (int k = 1; k < FEW_WAVES; ++k) v += sum[k][lane];
    const int n = n0 + 4 * q;
    if (c >= M || n >= N || at_a < 0) return;
    auto out = [&](auto zero) {
        using T = decltype(zero);
        const T t[4] = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        put<4>(static_cast<T*>(g.y) + (int64_t)(p0 + c) * g.ldy + n, N - n, t);
    };
    if (g.type == FOBQ_F32) out(0.f);
    else if (g.type == FOBQ_BF16) out((bf16_t)0.f);
    else out((f16_t)0.f);
}

// How many packed rows an expert has is known on the device only; the rules take their average over the experts that can have any, and half a tile more
// for the last one of each.  The measurements behind them (bf16, a scale per 128 x 128 unless it says otherwise, us; rows: the average of an expert):
//   16, 64 x 64, 64 x 128    1 token to 2 of 8 experts of 4096 x 4096: 9.6, 12.3, 13.1; 8 to 3 of 7 of 1000 x 2304: 7.2, 8.3, 8.8; 32: 10.2, 8.4, 10.3;
//                            8 to 4 of 64 of 1024 x 2048: 15.6, 11.4, 11.2; 32 to 8 of 128 of 2048 x 2048: 132, 84, 80 (memory)
//   64 x 64, 64 x 128        7 experts of 1000 x 2304, 143 rows: 12.6, 13.6; 439 rows: 23.3, 18.8
//   64 x 64, its blocks dealt to one set of wavefronts, to two   bf16, 7 experts of 1000 x k, 14 rows, k 1024, 1536, 2304, 4096: 5.7, 6.7, 8.1, 11.4 and 6.0, 6.8, 7.9, 10.7; 8 of
//                            1024 x k, 64 rows, k 1024, 1536, 2048, 2304: 6.9, 8.0, 9.2, 9.8 and 6.9, 7.9, 8.9, 9.4 (k 4096: no difference); more tiles than compute units,
//                            4 of 3000 x k, 83 rows, k 1024, 2304, 4096: 8.0, 12.3, 18.0 and 8.8, 13.4, 19.0; fp32 and a scale per row, 7 of 1000 x k, 143 rows, k 512,
//                            1024, 1536, 2304: 9.0, 13.0, 16.4, 21.4 and 10.5, 12.9, 15.5, 19.6; 8 of 1024 x k, 64 rows, k 512, 1024, 2304: 7.3, 9.7, 15.3 and 7.5, 9.3, 13.3
//   64 x 128, 128 x 256, 256 x 256   64 experts of 4096 x 2048, 128 rows: 181, 150, 176; 512 rows: 530, 410, 381; 8 of 4096 x 4096, 83 rows: 29, 35, 45;
//                            256 rows: 64, 69, 58; 1024 rows: 219, 181, 178; 64 of 1024 x 2048, 256 rows: 71, 63, 66
//   fp32, 64 x 128, 128 x 128, 128 x 256   8 of 4096 x 4096, 1024 rows: 365, 321, 352; 128 of 2048 x 2048, 64 rows: 168, 170, 166
// The larger ones are chosen by rounds of workgroups (two of 64 x 128 or 128 x 128 on a compute unit at a time, one of the others), a round of 128 x 256
// taking 1.45 times as long as one of 64 x 128, 1.57 with a scale per row of B, one of 256 x 256 2.45 times, one of 128 x 128 in fp32 1.6 times.
ExpertPlan expert_plan(int cus, int64_t rows, int experts, int64_t n, int64_t k, int type, int per)
{
    const int64_t with_rows = std::min<int64_t>(rows, experts);
    auto tiles = [&](int tm, int tn) { return std::max(with_rows, rows / tm + with_rows / 2) * ((n + tn - 1) / tn); };
    auto rounds = [&](int tm, int tn, int at_once) { return (double)((tiles(tm, tn) + at_once * cus - 1) / (at_once * cus)); };
    ExpertPlan p;
    p.parts = 1;
    if (rows <= 8 * with_rows && tiles(64, 64) < cus) {
        p.tm = p.tn = 16;
    } else if (tiles(64, 128) < cus) {
        p.tm = p.tn = 64;
        if (k >= 2048 && 2 * tiles(64, 64) <= (type == FOBQ_F32 ? 3 : 2) * cus) p.parts = 2;
    } else {
        p.tm = 64;
        p.tn = 128;
        double best = rounds(64, 128, 2);
        auto consider = [&](int tm, int tn, int at_once, double cost) {
            if (cost * rounds(tm, tn, at_once) < best) p.tm = tm, p.tn = tn, best = cost * rounds(tm, tn, at_once);
        };
        if (type == FOBQ_F32) consider(128, 128, 2, 1.6);
        else consider(128, 256, 1, per == 128 ? 1.45 : 1.57);
        if (type != FOBQ_F32 && per == 128) consider(256, 256, 1, 2.45);
    }
    // Each expert with rows has at least one tile, and one more for every tm rows further.
    p.tiles = (with_rows + (rows - with_rows) / p.tm) * ((n + p.tn - 1) / p.tn);
    return p;
}

template <int FA, int FB, int PER>
static hipError_t experts_of(hipStream_t s, const ExpertPlan& p, const ExpertView& g)
{
    const dim3 grid((unsigned)p.tiles);
    const bool exact = g.type == FOBQ_F32;
    if (p.tm == 16) {
        hipLaunchKernelGGL((fp8_experts_few_kernel<FA, FB, PER>), grid, dim3(64 * FEW_WAVES), 0, s, g);
    } else if (p.tm == 64 && p.tn == 64) {
        if (p.parts == 2) {
            if (exact) hipLaunchKernelGGL((fp8_experts_kernel<64, 64, 2, 2, 2, 2, FA, FB, PER, true>), grid, dim3(512), 0, s, g);
            else hipLaunchKernelGGL((fp8_experts_kernel<64, 64, 2, 2, 2, 2, FA, FB, PER, false>), grid, dim3(512), 0, s, g);
        } else {
            if (exact) hipLaunchKernelGGL((fp8_experts_kernel<64, 64, 2, 2, 4, 1, FA, FB, PER, true>), grid, dim3(256), 0, s, g);
            else hipLaunchKernelGGL((fp8_experts_kernel<64, 64, 2, 2, 4, 1, FA, FB, PER, false>), grid, dim3(256), 0, s, g);
        }
    } else if (p.tm == 64) {
        if (exact) hipLaunchKernelGGL((fp8_experts_kernel<64, 128, 1, 4, 3, 1, FA, FB, PER, true>), grid, dim3(256), 0, s, g);
        else hipLaunchKernelGGL((fp8_experts_kernel<64, 128, 1, 4, 3, 1, FA, FB, PER, false>), grid, dim3(256), 0, s, g);
    } else if (exact) {
        hipLaunchKernelGGL((fp8_experts_kernel<128, 128, 2, 2, 2, 1, FA, FB, PER, true>), grid, dim3(256), 0, s, g);
    } else if (p.tm == 128) {
        hipLaunchKernelGGL((fp8_experts_kernel<128, 256, 2, 4, 3, 1, FA, FB, PER, false>), grid, dim3(512), 0, s, g);
    } else {
        if constexpr (PER == 128) hipLaunchKernelGGL((fp8_experts_kernel<256, 256, 2, 4, 2, 1, FA, FB, PER, false>), grid, dim3(512), 0, s, g);
    }
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
