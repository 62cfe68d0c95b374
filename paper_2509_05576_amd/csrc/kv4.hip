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

namespace fobq {

constexpr float KV4_TINY = 1.17549435e-38f;   // 2^-126: the smallest scale, and what a row of zeros gets

// Where ROWS packed rows from `row0` on lie in the cache: row numbers of head 0, or -1.  One search for the first; a row that is not of
// the same sequence is searched for by itself.
template <int ROWS>
__device__ __forceinline__ void kv4_rows_of(const Kv4View& c, const Kv4Seqs& s, int row0, int64_t (&at)[ROWS])
{
    auto begins = [&](int i) { return (int64_t)kv4_rows(s.starts, i, s.rows).first; };
    int b = s.starts ? wave_search(s.n_seqs, row0, begins) : row0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int row = row0 + r;
        at[r] = -1;
        if (row >= s.rows || (!s.starts && row >= s.n_seqs)) continue;      // (without starts, row i is sequence i's)
        if (r > 0) {
            // (several sequences may begin at a row: the last of them has it, the others are empty)
            const Kv4Rows mine = kv4_rows(s.starts, b, s.rows);
            if (row >= mine.first + mine.count && b + 1 < s.n_seqs) b = s.starts ? wave_search(s.n_seqs, row, begins) : row;
        }
        const Kv4Place p = kv4_place(s, c.pages, c.shift, b, row);
        if (p.page >= 0) at[r] = (((int64_t)p.page * c.heads) << c.shift) + p.place;
    }
}

// A wavefront has ROWS packed rows: its lanes go through the heads' rows of keys (blockIdx.y = 0) or values, 64 / (dim / 8) heads at a time.
template <class T, int DIM, int ROWS>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4View c, Kv4Seqs s, const T* __restrict__ k, int64_t k_row, int64_t k_head,
                                                         const T* __restrict__ v, int64_t v_row, int64_t v_head)
{
    constexpr int LANES = DIM / 8, AT_ONCE = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const int row0 = __builtin_amdgcn_readfirstlane((blockIdx.x * 4 + (threadIdx.x >> 6)) * ROWS);
    if (row0 >= s.rows) return;
    const bool values = blockIdx.y != 0;
    const T* __restrict__ src = values ? v + (int64_t)row0 * v_row : k + (int64_t)row0 * k_row;
    const int64_t row_ld = values ? v_row : k_row, head_ld = values ? v_head : k_head;
    uint8_t* __restrict__ codes = values ? c.v_codes : c.k_codes;
    uint32_t* __restrict__ grids = values ? c.v_grids : c.k_grids;
    const int part = lane % LANES;
    int64_t first[ROWS];
    kv4_rows_of<ROWS>(c, s, row0, first);
    for (int h0 = 0; h0 < c.heads; h0 += AT_ONCE) {
        const int h = h0 + lane / LANES;
        float x[ROWS][8];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[r][i] = 0.f;
            if (h < c.heads && first[r] >= 0) load8(src + r * row_ld + h * head_ld + 8 * part, x[r]);
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float lo = 0.f, hi = 0.f, bad = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lo = fminf(lo, x[r][i]);
                hi = fmaxf(hi, x[r][i]);
                bad = fmaf(x[r][i], 0.f, bad);          // NaN as soon as one of them is not finite
            }
#pragma unroll
            for (int off = LANES / 2; off > 0; off >>= 1) {
                lo = fminf(lo, __shfl_xor(lo, off));
                hi = fmaxf(hi, __shfl_xor(hi, off));
                bad += __shfl_xor(bad, off);
            }
            if (h >= c.heads || first[r] < 0) continue;
            const float range = (hi - lo) / 15.f;
            float scale = __uint_as_float((__float_as_uint(range) + 0xffffu) & 0xffff0000u);
            scale = fmaxf(scale, KV4_TINY);
            uint32_t word = 0;
            uint32_t grid = 0x7fc00000u;             // a row that is not finite, or whose range is not: NaN throughout
            if (bad == 0.f && range <= 3.4028235e38f) {
                const float inv = 1.f / scale;
                auto level = [&](float v) {                // rint(v / scale)
                    const float y = v * inv;
                    return rintf(fmaf(fmaf(-y, scale, v), inv, y));
                };
                const float zero = fminf(fmaxf(level(-lo), 0.f), 15.f);
                grid = __float_as_uint(scale) | (uint32_t)zero;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float q = fminf(fmaxf(level(x[r][i]) + zero, 0.f), 15.f);
                    word |= (uint32_t)q << (4 * i);
                }
            }
            const int64_t at = first[r] + ((int64_t)h << c.shift);
            *reinterpret_cast<uint32_t*>(codes + at * (DIM / 2) + 4 * part) = word;
            if (part == 0) grids[at] = grid;
        }
    }
}

// The same rows back as the values they stand for, scale * (code - zero), rounded to T once.  Tokens on no page of the cache read 0.
template <class T, int DIM, int ROWS>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4View c, Kv4Seqs s, T* __restrict__ k, int64_t k_row, int64_t k_head,
                                                       T* __restrict__ v, int64_t v_row, int64_t v_head)
{
    constexpr int LANES = DIM / 8, AT_ONCE = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const int row0 = __builtin_amdgcn_readfirstlane((blockIdx.x * 4 + (threadIdx.x >> 6)) * ROWS);
    const Kv4Rows final = kv4_rows(s.starts, s.n_seqs - 1, s.rows);
    const int rows = min(ROWS, (s.starts ? final.first + final.count : min(s.rows, s.n_seqs)) - row0);     // not behind the last sequence
    if (rows <= 0) return;
    const bool values = blockIdx.y != 0;
    T* __restrict__ dst = values ? v + (int64_t)row0 * v_row : k + (int64_t)row0 * k_row;
    const int64_t row_ld = values ? v_row : k_row, head_ld = values ? v_head : k_head;
    const uint8_t* __restrict__ codes = values ? c.v_codes : c.k_codes;
    const uint32_t* __restrict__ grids = values ? c.v_grids : c.k_grids;
    const int part = lane % LANES;
    int64_t first[ROWS];
    kv4_rows_of<ROWS>(c, s, row0, first);
    for (int h = lane / LANES; h < c.heads; h += AT_ONCE) {
        uint32_t word[ROWS], grid[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            word[r] = grid[r] = 0;
            if (first[r] < 0) continue;
            const int64_t at = first[r] + ((int64_t)h << c.shift);
            word[r] = *reinterpret_cast<const uint32_t*>(codes + at * (DIM / 2) + 4 * part);
            grid[r] = grids[at];
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (r >= rows) continue;
            const float scale = __uint_as_float(grid[r] & 0xffff0000u), zero = (float)kv4_zero(grid[r]);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = scale * ((float)(word[r] >> (4 * i) & 15u) - zero);
            store8(dst + r * row_ld + h * head_ld + 8 * part, x);
        }
    }
}

// Rows of a wavefront: four where there are enough of them to fill the chip all the same.  A wavefront's time is the latency of finding its
// rows; 16000 rows of 8 x 128 channels take AAA us to append and read with one, BBB with four.
constexpr int KV4_MANY_ROWS = 4096;

template <class T, int DIM>
static void append_of(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, const T* k, int64_t k_row, int64_t k_head, const T* v, int64_t v_row, int64_t v_head)
{
    if (s.rows < KV4_MANY_ROWS)
        hipLaunchKernelGGL((kv4_append_kernel<T, DIM, 1>), dim3((unsigned)((s.rows + 3) / 4), 2), dim3(256), 0, st, c, s, k, k_row, k_head, v, v_row, v_head);
    else
        hipLaunchKernelGGL((kv4_append_kernel<T, DIM, 4>), dim3((unsigned)((s.rows + 15) / 16), 2), dim3(256), 0, st, c, s, k, k_row, k_head, v, v_row, v_head);
}
template <class T>
static hipError_t append_of(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, const void* kp, int64_t k_row, int64_t k_head, const void* vp, int64_t v_row,
                            int64_t v_head)
{
    const T *k = static_cast<const T*>(kp), *v = static_cast<const T*>(vp);
    if (c.dim == 64) append_of<T, 64>(st, c, s, k, k_row, k_head, v, v_row, v_head);
    else if (c.dim == 128) append_of<T, 128>(st, c, s, k, k_row, k_head, v, v_row, v_head);
    else append_of<T, 256>(st, c, s, k, k_row, k_head, v, v_row, v_head);
    return hipGetLastError();
}

template <class T, int DIM>
static void read_of(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, T* k, int64_t k_row, int64_t k_head, T* v, int64_t v_row, int64_t v_head)
{
    if (s.rows < KV4_MANY_ROWS)
        hipLaunchKernelGGL((kv4_read_kernel<T, DIM, 1>), dim3((unsigned)((s.rows + 3) / 4), 2), dim3(256), 0, st, c, s, k, k_row, k_head, v, v_row, v_head);
    else
        hipLaunchKernelGGL((kv4_read_kernel<T, DIM, 4>), dim3((unsigned)((s.rows + 15) / 16), 2), dim3(256), 0, st, c, s, k, k_row, k_head, v, v_row, v_head);
}
template <class T>
static hipError_t read_of(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, void* kp, int64_t k_row, int64_t k_head, void* vp, int64_t v_row, int64_t v_head)
{
    T *k = static_cast<T*>(kp), *v = static_cast<T*>(vp);
    if (c.dim == 64) read_of<T, 64>(st, c, s, k, k_row, k_head, v, v_row, v_head);
    else if (c.dim == 128) read_of<T, 128>(st, c, s, k, k_row, k_head, v, v_row, v_head);
    else read_of<T, 256>(st, c, s, k, k_row, k_head, v, v_row, v_head);
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
