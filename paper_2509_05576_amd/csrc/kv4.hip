// Rows of the 4-bit cache: new keys and values onto their grids (append) and back (read).
//
// Every row of a head's `dim` channels has a grid of 16 levels of its own, the layers' min-max grid at 4 bits (Section 3): lo =
// min(min x, 0), hi = max(max x, 0), scale = (hi - lo) / 15, zero = rint(-lo / scale), code = clamp(rint(x / scale) + zero, 0, 15).
// The scale is held in bf16 and rounded up to it, so that 15 steps still reach from lo to hi, and codes and zero are taken against
// the scale as held.  The inputs have at most 11 bits and the scale 8, so that a quotient that is not on the border of two levels is at
// least 2^-20 away from it: the reciprocal's product, corrected by its remainder (an fma's, exact), falls on the same side, and on
// the border where the exact one does.  (The language's division takes four times the instructions: 16000 rows of 8 x 128 channels
// were bound by them.)
//
// Memory bound: a lane has 8 channels of a row, 16 bytes in, one word of codes out; dim / 8 lanes share a row and its minimum and
// maximum by shuffles.
#include "kv4.h"

#include <type_traits>

namespace fobq {

constexpr float KV4_TINY = 1.17549435e-38f;   // 2^-126: the smallest scale, and what a row of zeros gets

// Where packed row `row` lies in the cache: the row number of head 0, or -1.
__device__ __forceinline__ int64_t kv4_row_of(const Kv4View& c, const Kv4Seqs& s, int row)
{
    if (!s.starts && row >= s.n_seqs) return -1;             // (without starts, row i is sequence i's)
    // several sequences may begin at this row: the last of them has it, the others are empty
    const int b = s.starts ? wave_search(s.n_seqs, row, [&](int i) { return (int64_t)kv4_rows(s.starts, i, s.rows).first; }) : row;
    const Kv4Place p = kv4_place(s, c.pages, c.shift, b, row);
    return p.page < 0 ? -1 : (((int64_t)p.page * c.heads) << c.shift) + p.place;
}

// f over groups of 8, 16 or 32 lanes, the result in all of them: the neighbour, the other pair, the other half of eight, of sixteen, of
// thirty-two, as operands of the instruction (through LDS, as the language's shuffles go, this was most of the kernel).
template <int LANES, class F>
__device__ __forceinline__ float over_lanes(float x, F f)
{
    auto dpp = [](float v, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
    x = f(x, dpp(x, std::integral_constant<int, 0xB1>()));
    x = f(x, dpp(x, std::integral_constant<int, 0x4E>()));
    x = f(x, dpp(x, std::integral_constant<int, 0x141>()));
    if constexpr (LANES > 8) x = f(x, dpp(x, std::integral_constant<int, 0x140>()));
    if constexpr (LANES > 16) {
        const uint32_t u = __float_as_uint(x);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return x;
}

// A wavefront has a packed row: its lanes go through the heads' rows of keys (blockIdx.y = 0) or values, 64 / (dim / 8) heads at a time.
// (16000 rows of 8 heads of 128 channels, bf16: 23 us, 3.7 TB/s, by vector instructions and memory alike; four rows a wavefront took longer.)
template <class T, int DIM>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4View c, Kv4Seqs s, const T* __restrict__ k, int64_t k_row, int64_t k_head,
                                                         const T* __restrict__ v, int64_t v_row, int64_t v_head)
{
    constexpr int LANES = DIM / 8, AT_ONCE = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (row >= s.rows) return;
    const bool values = blockIdx.y != 0;
    const int64_t first = kv4_row_of(c, s, row);
    if (first < 0) return;
    const T* __restrict__ src = values ? v + (int64_t)row * v_row : k + (int64_t)row * k_row;
    const int64_t head_ld = values ? v_head : k_head;
    uint8_t* __restrict__ codes = values ? c.v_codes : c.k_codes;
    uint32_t* __restrict__ grids = values ? c.v_grids : c.k_grids;
    const int part = lane % LANES;
    for (int h0 = 0; h0 < c.heads; h0 += AT_ONCE) {
        const int h = h0 + lane / LANES;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (h < c.heads) load8(src + h * head_ld + 8 * part, x);
        float lo = 0.f, hi = 0.f, bad = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
            bad = fmaf(x[i], 0.f, bad);                       // NaN as soon as one of them is not finite
        }
        lo = over_lanes<LANES>(lo, [](float a, float b) { return fminf(a, b); });
        hi = over_lanes<LANES>(hi, [](float a, float b) { return fmaxf(a, b); });
        bad = over_lanes<LANES>(bad, [](float a, float b) { return a + b; });
        if (h >= c.heads) continue;
        // the range, rounded up: next to an end of 15 bf16 steps the other end may be too small for fp32 to add, and counts all the same
        float range = hi - lo;
        const float larger = fmaxf(hi, -lo);
        if (fminf(hi, -lo) > range - larger) range = __uint_as_float(__float_as_uint(range) + 1);
        range /= 15.f;
        float scale = __uint_as_float((__float_as_uint(range) + 0xffffu) & 0xffff0000u);
        scale = fmaxf(scale, KV4_TINY);
        uint32_t word = 0;
        uint32_t grid = 0x7fc00000u;                          // a row that is not finite, or whose range is not: NaN throughout
        if (bad == 0.f && range <= 3.4028235e38f) {
            const float inv = 1.f / scale;
            auto level = [&](float v) {                       // rint(v / scale)
                const float y = v * inv;
                return rintf(fmaf(fmaf(-y, scale, v), inv, y));
            };
            const float zero = fminf(fmaxf(level(-lo), 0.f), 15.f);
            grid = __float_as_uint(scale) | (uint32_t)zero;
#pragma unroll
            for (int i = 0; i < 8; ++i) word |= (uint32_t)fminf(fmaxf(level(x[i]) + zero, 0.f), 15.f) << (4 * i);
        }
        const int64_t at = first + ((int64_t)h << c.shift);
        *reinterpret_cast<uint32_t*>(codes + at * (DIM / 2) + 4 * part) = word;
        if (part == 0) grids[at] = grid;
    }
}

// The same rows back as the values they stand for, scale * (code - zero), rounded to T once.  Tokens on no page of the cache read 0.
// (The same rows: 16 us, 5.3 TB/s.)
template <class T, int DIM>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4View c, Kv4Seqs s, T* __restrict__ k, int64_t k_row, int64_t k_head,
                                                       T* __restrict__ v, int64_t v_row, int64_t v_head)
{
    constexpr int LANES = DIM / 8, AT_ONCE = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const Kv4Rows final = kv4_rows(s.starts, s.n_seqs - 1, s.rows);
    if (row >= (s.starts ? final.first + final.count : min(s.rows, s.n_seqs))) return;      // behind the last sequence
    const bool values = blockIdx.y != 0;
    const int64_t first = kv4_row_of(c, s, row);
    T* __restrict__ dst = values ? v + (int64_t)row * v_row : k + (int64_t)row * k_row;
    const int64_t head_ld = values ? v_head : k_head;
    const uint8_t* __restrict__ codes = values ? c.v_codes : c.k_codes;
    const uint32_t* __restrict__ grids = values ? c.v_grids : c.k_grids;
    const int part = lane % LANES;
    for (int h = lane / LANES; h < c.heads; h += AT_ONCE) {
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (first >= 0) {
            const int64_t at = first + ((int64_t)h << c.shift);
            const uint32_t word = *reinterpret_cast<const uint32_t*>(codes + at * (DIM / 2) + 4 * part), grid = grids[at];
            const float scale = __uint_as_float(grid & 0xffff0000u), zero = (float)kv4_zero(grid);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = scale * ((float)(word >> (4 * i) & 15u) - zero);
        }
        store8(dst + h * head_ld + 8 * part, x);
    }
}

template <class T>
static hipError_t append_of(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row,
                            int64_t v_head)
{
    const dim3 grid((unsigned)((s.rows + 3) / 4), 2), block(256);
    const T *kt = static_cast<const T*>(k), *vt = static_cast<const T*>(v);
    if (c.dim == 64) hipLaunchKernelGGL((kv4_append_kernel<T, 64>), grid, block, 0, st, c, s, kt, k_row, k_head, vt, v_row, v_head);
    else if (c.dim == 128) hipLaunchKernelGGL((kv4_append_kernel<T, 128>), grid, block, 0, st, c, s, kt, k_row, k_head, vt, v_row, v_head);
    else hipLaunchKernelGGL((kv4_append_kernel<T, 256>), grid, block, 0, st, c, s, kt, k_row, k_head, vt, v_row, v_head);
    return hipGetLastError();
}

template <class T>
static hipError_t read_of(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, void* k, int64_t k_row, int64_t k_head, void* v, int64_t v_row, int64_t v_head)
{
    const dim3 grid((unsigned)((s.rows + 3) / 4), 2), block(256);
    T *kt = static_cast<T*>(k), *vt = static_cast<T*>(v);
    if (c.dim == 64) hipLaunchKernelGGL((kv4_read_kernel<T, 64>), grid, block, 0, st, c, s, kt, k_row, k_head, vt, v_row, v_head);
    else if (c.dim == 128) hipLaunchKernelGGL((kv4_read_kernel<T, 128>), grid, block, 0, st, c, s, kt, k_row, k_head, vt, v_row, v_head);
    else hipLaunchKernelGGL((kv4_read_kernel<T, 256>), grid, block, 0, st, c, s, kt, k_row, k_head, vt, v_row, v_head);
    return hipGetLastError();
}

hipError_t launch_kv4_append(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, int type, const void* k, int64_t k_row, int64_t k_head, const void* v,
                             int64_t v_row, int64_t v_head)
{
    return type == FOBQ_BF16 ? append_of<bf16_t>(st, c, s, k, k_row, k_head, v, v_row, v_head) : append_of<f16_t>(st, c, s, k, k_row, k_head, v, v_row, v_head);
}

hipError_t launch_kv4_read(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, int type, void* k, int64_t k_row, int64_t k_head, void* v, int64_t v_row,
                           int64_t v_head)
{
    if (type == FOBQ_F32) return read_of<float>(st, c, s, k, k_row, k_head, v, v_row, v_head);
    return type == FOBQ_BF16 ? read_of<bf16_t>(st, c, s, k, k_row, k_head, v, v_row, v_head) : read_of<f16_t>(st, c, s, k, k_row, k_head, v, v_row, v_head);
}

}  // namespace fobq
