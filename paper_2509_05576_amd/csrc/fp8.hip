// Matrices in 8-bit floating point with a scale for each block of 128 columns and 1 or 128 rows: from 16- and 32-bit matrices, and
// from the codes of a quantized layer.
//
// A block's scale is its largest magnitude over the type's largest value (e4m3 448, e5m2 57344), at least 2^-126 (which a block of
// zeros has); the values are the nearest ones to x / scale, ties to even.  A block that holds an Inf or NaN is NaN throughout.
// The quotient: with top = 0.875 * 2^9 or * 2^16, x / (most / top) = (0.875 x) / (most / 2^9 or 2^16); one multiplication by the reciprocal
// and one correction from the remainder round it to fp32 as a division would.  Where that lies on the border of two 8-bit values (one of 2^20
// fp32 quotients, and zeros) the remainder says on which side the quotient lies, so that it is rounded to 8 bits once and not twice.  It
// never passes the largest value by more than a rounding, which the conversion takes back.  The remainder has bits 2^-47 below x: blocks
// whose largest is below 2^-40 are taken 2^80 times as large on both sides, so that those are not below what fp32 holds for any x that does not
// round to 0 (that is, above 2^-33 of the largest).
#include "lowbit.h"

namespace fobq {

constexpr float FP8_TINY = 1.17549435e-38f;

template <int FORMAT> struct Fp8;          // fobq_fp8
template <> struct Fp8<FOBQ_E4M3> { static constexpr float TOP = 448.f, POW = 1.f / 512; };
template <> struct Fp8<FOBQ_E5M2> { static constexpr float TOP = 57344.f, POW = 1.f / 65536; };

template <int FORMAT>
__device__ __forceinline__ uint32_t to_fp8x4(float a, float b, float c, float d)
{
    int w = 0;
    if constexpr (FORMAT == FOBQ_E4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    }
    return (uint32_t)w;
}

// what turns a block's values into 8-bit ones
struct Fp8Scale { float scale, pre, most, inv, corr; };
template <int FORMAT>
__device__ __forceinline__ Fp8Scale fp8_scale(uint32_t bits)
{
    const float most = __uint_as_float(bits), scale = most / Fp8<FORMAT>::TOP;
    if (bits >= 0x7f800000u) return Fp8Scale{__builtin_nanf(""), __builtin_nanf(""), 0.f, 1.f, 0.f};
    if (scale < FP8_TINY) return Fp8Scale{FP8_TINY, 1.f, 0.f, 0x1p126f, 0.f};
    const float lift = most < 0x1p-40f ? 0x1p80f : 1.f, m = most * lift * Fp8<FORMAT>::POW, inv = 1.f / m;
    return Fp8Scale{scale, 0.875f * lift, m, inv, inv};
}
// x / scale, rounded once: the remainder of the first guess is exact (its product's error is taken along, and what is left of x fits)
__device__ __forceinline__ float fp8_quotient(const Fp8Scale& s, float x)
{
    const float y = x * s.pre * s.inv, p = y * s.most, e = fmaf(y, s.most, -p);
    return fmaf(fmaf(x, s.pre, -p) - e, s.corr, y);
}
// A quotient y that lies on a border, or not: one step to the side on which x / scale lies if that is not y itself.  (The remainder's sign is
// exact; an odd fp32 number is on no border, nor is 0, which a value far below the smallest one gives.)
__device__ __forceinline__ float fp8_side(const Fp8Scale& s, float x, float y)
{
    const float p = y * s.most, rest = fmaf(x, s.pre, -p) - fmaf(y, s.most, -p);
    const uint32_t bits = __float_as_uint(y);
    if (s.most == 0.f || rest == 0.f || (bits & 1) || bits << 1 == 0) return y;          // (most 0: y is exact, or NaN)
    return __uint_as_float(bits + ((rest > 0.f) == (y > 0.f) ? 1 : -1));
}

// 16 adjacent values of a row, or those of them that the row has (0 behind them).  As they are: where they were made floats here, the
// branch waited for them, and a thread's next load for that.
template <class T>
__device__ __forceinline__ void get16(const T* __restrict__ src, int left, T* x)
{
    if (left >= 16) {
        __builtin_memcpy(x, src, 16 * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = i < left ? src[i] : (T)0.f;
    }
}
// their 8-bit values into the row
template <class T, int FORMAT>
__device__ __forceinline__ void put16(uint8_t* __restrict__ dst, int left, const Fp8Scale& s, const T* x)
{
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = fp8_quotient(s, (float)x[i]);
    // a border has no lower bits than 2^-4 (e5m2: 2^-3) of its value's highest
    uint32_t low = ~0u;
#pragma unroll
    for (int i = 0; i < 16; ++i) low = min(low, __float_as_uint(y[i]) << 13);
    if (low == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = fp8_side(s, (float)x[i], y[i]);
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = to_fp8x4<FORMAT>(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    if (left >= 16) {
        __builtin_memcpy(__builtin_assume_aligned(dst, 16), w, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < left) dst[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}
// the largest magnitude as its bits, which order as the magnitudes do, Inf and NaN above all others
template <class T>
__device__ __forceinline__ uint32_t most16(const T* x)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint((float)x[i]) & 0x7fffffffu);
    return m;
}
// over eight lanes: the neighbour, the other pair, the other half
__device__ __forceinline__ uint32_t most_of_8(uint32_t m)
{
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, true));
}

// Item first + i of rows of `pieces` items: its row and its place there.  `first` is the workgroup's: one 64-bit division for all of its
// threads, and a 32-bit one each.
struct Item { int64_t row; int piece; };
__device__ __forceinline__ Item item_of(int64_t first, unsigned i, unsigned pieces)
{
    const int64_t row = first / pieces;
    const unsigned at = (unsigned)(first - row * pieces) + i, rows = at / pieces;
    return Item{row + rows, (int)(at - rows * pieces)};
}

// A scale per row: 8 lanes have a block, 16 columns each; a wavefront eight consecutive blocks of a row.  (8192 x 8192: bf16 50 us, 4.1 TB/s;
// fp32 60 us, 5.6 TB/s, as memory has it.  With 8 columns a lane, half the loads in flight and stores of 8 bytes: 62 and 68.)
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void fp8_rows_kernel(const T* __restrict__ x, int64_t ld, Fp8View out)
{
    const int lane = threadIdx.x & 63;
    const Item at = item_of((int64_t)blockIdx.x * 4, threadIdx.x >> 6, (out.cols + 1023) / 1024);
    const int64_t row = at.row;
    const int col = at.piece * 1024 + 16 * lane, left = out.cols - col;
    if (row >= out.rows) return;
    T v[16];
    get16(x + row * ld + col, left, v);
    const Fp8Scale s = fp8_scale<FORMAT>(most_of_8(most16(v)));
    put16<T, FORMAT>(out.values + row * out.ld + col, left, s, v);
    if ((lane & 7) == 0 && left > 0) out.scales[(int64_t)(col / 128) * out.ld_scales + row] = s.scale;
}

// A scale per 128 rows: a workgroup has a block of 128 x 128, 64 values a thread, which stay in registers between the two passes.
// (8192 x 8192: fp32 60 us, 5.6 TB/s; bf16 52 us, 3.9 TB/s.)
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void fp8_tiles_kernel(const T* __restrict__ x, int64_t ld, Fp8View out)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const unsigned across = (out.cols + 127) / 128, down = blockIdx.x / across, over = blockIdx.x - down * across;
    const int col = over * 128 + 16 * (tid & 7), left = out.cols - col;
    const int64_t row0 = (int64_t)down * 128 + (tid >> 3);
    __shared__ uint32_t part[4];
    T v[4][16];
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t row = row0 + 32 * k;
        get16(x + row * ld + col, row < out.rows ? left : 0, v[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) most = max(most, most16(v[k]));
    most = most_of_8(most);
#pragma unroll
    for (int off = 32; off > 4; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off));
    if (lane == 0) part[tid >> 6] = most;
    __syncthreads();
    most = max(max(part[0], part[1]), max(part[2], part[3]));
    const Fp8Scale s = fp8_scale<FORMAT>(most);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t row = row0 + 32 * k;
        if (row < out.rows) put16<T, FORMAT>(out.values + row * out.ld + col, left, s, v[k]);
    }
    if (tid == 0) out.scales[(int64_t)over * out.ld_scales + down] = s.scale;
}

// The codes of a layer (Section 3: q = scale (code - zero)): code - zero is an integer of at most 15 in magnitude for codes of up to
// four bits, which e4m3 holds exactly, and the grid's scale is the block's.  16 codes a thread; the last workgroups turn the scales from
// rows x groups into blocks x rows, a row a lane (written beside the codes, one word in a line at a time, they took longer than those).  (8192 x 8192: 22 us, 6.2 TB/s.)
__global__ __launch_bounds__(256) void fp8_codes_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales, const float* __restrict__ zeros,
                                                        int groups, int group, unsigned code_wgs, Fp8View out)
{
    if (blockIdx.x >= code_wgs) {
        const Item at = item_of((int64_t)(blockIdx.x - code_wgs) * 256, threadIdx.x, out.rows);
        const int64_t kb = at.row;
        if (kb * 128 < out.cols) out.scales[kb * out.ld_scales + at.piece] = scales[(int64_t)at.piece * groups + (group ? kb * 128 / group : 0)];
        return;
    }
    const Item at = item_of((int64_t)blockIdx.x * 256, threadIdx.x, (out.cols + 15) / 16);
    const int64_t row = at.row;
    const int col = at.piece * 16, left = out.cols - col;
    if (row >= out.rows) return;
    const float zero = zeros[row * groups + (group ? col / group : 0)];
    const uint8_t* __restrict__ src = codes + row * out.cols + col;
    uint8_t* dst = out.values + row * out.ld + col;
    auto four = [&](uint32_t w) {
        return to_fp8x4<FOBQ_E4M3>((float)(w & 255u) - zero, (float)(w >> 8 & 255u) - zero, (float)(w >> 16 & 255u) - zero, (float)(w >> 24) - zero);
    };
    if (left >= 16) {
        uint32_t w[4];
        __builtin_memcpy(w, src, 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = four(w[k]);
        __builtin_memcpy(dst, w, 16);
    } else {
        for (int i = 0; i < left; ++i) dst[i] = (uint8_t)four(src[i]);
    }
}

template <class T, int FORMAT>
static hipError_t quantize_of(hipStream_t s, const void* x, int64_t ld, const Fp8View& out)
{
    const int blocks = (out.cols + 127) / 128;
    if (out.per == 1) {
        const int64_t items = (int64_t)out.rows * ((blocks + 7) / 8);
        hipLaunchKernelGGL((fp8_rows_kernel<T, FORMAT>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, static_cast<const T*>(x), ld, out);
    } else {
        hipLaunchKernelGGL((fp8_tiles_kernel<T, FORMAT>), dim3((unsigned)((int64_t)blocks * ((out.rows + 127) / 128))), dim3(256), 0, s, static_cast<const T*>(x), ld, out);
    }
    return hipGetLastError();
}

hipError_t launch_fp8_quantize(hipStream_t s, const void* x, int type, int64_t ld, const Fp8View& out)
{
    const bool e4 = out.format == FOBQ_E4M3;
    if (type == FOBQ_F32) return e4 ? quantize_of<float, FOBQ_E4M3>(s, x, ld, out) : quantize_of<float, FOBQ_E5M2>(s, x, ld, out);
    if (type == FOBQ_BF16) return e4 ? quantize_of<bf16_t, FOBQ_E4M3>(s, x, ld, out) : quantize_of<bf16_t, FOBQ_E5M2>(s, x, ld, out);
    return e4 ? quantize_of<f16_t, FOBQ_E4M3>(s, x, ld, out) : quantize_of<f16_t, FOBQ_E5M2>(s, x, ld, out);
}

hipError_t launch_fp8_from_codes(hipStream_t s, const uint8_t* codes, const float* scales, const float* zeros, int group, const Fp8View& out)
{
    const int64_t pieces = (int64_t)out.rows * ((out.cols + 15) / 16), blocks = (int64_t)out.rows * ((out.cols + 127) / 128);
    const unsigned code_wgs = (unsigned)((pieces + 255) / 256);
    hipLaunchKernelGGL(fp8_codes_kernel, dim3(code_wgs + (unsigned)((blocks + 255) / 256)), dim3(256), 0, s, codes, scales, zeros,
                       group ? out.cols / group : 1, group, code_wgs, out);
    return hipGetLastError();
}

}  // namespace fobq
