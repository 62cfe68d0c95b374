// What stands in front of and between products of 8-bit blocks: the residual's addition with a root-mean-square norm, and the gated
// activation, both straight into blocks of 128 columns with a scale per row.
//
// Memory bound: a lane has 16 columns of a row, eight lanes a block, and everything between the loads and the 8-bit values stays in
// registers.  The sum of squares is in fp64, which no row of finite values passes, so that rows of very large and very small values lose nothing.
// What is rounded to 8 bits is a value's product with largest 8-bit value / largest of the block, one multiplication (fobq_fp8_quantize's quotient, rounded once, takes ten
// instructions and is for values that are given).  These values have been rounded to fp32 already, so that one in some 20000 (bf16 sums and weights, whose products often lie on
// a border) to a million (fp32) falls on the other side of an 8-bit border than in 64 bits.  A factor that all of a row's values share would round
// each of them once more and cancels out of a block: the norm keeps it out of them (in 3.3e8 values 10541 others than in 64 bits, with it 13733).
#include "fp8.h"

#include <type_traits>

namespace fobq {

// 16 values of a block as multiples of `unit`, most the largest multiple's magnitude's bits, into 8 bits; the block's scale
template <int FORMAT>
__device__ __forceinline__ float put16_by(uint8_t* __restrict__ dst, int left, uint32_t most, const float* y, float unit = 1.f)
{
    const float top = __uint_as_float(most), largest = top * unit, scale = largest / Fp8<FORMAT>::TOP;
    const bool fine = largest < __builtin_inff();
    const float by = !fine ? __builtin_nanf("") : scale < FP8_TINY ? 0x1p126f * unit : Fp8<FORMAT>::TOP / top;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = to_fp8x4<FORMAT>(y[4 * i] * by, y[4 * i + 1] * by, y[4 * i + 2] * by, y[4 * i + 3] * by);
    if (left >= 16) {
        __builtin_memcpy(__builtin_assume_aligned(dst, 16), w, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < left) dst[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
    return fine ? fmaxf(scale, FP8_TINY) : __builtin_nanf("");
}

// y as T into 16 adjacent places of a row
template <class T>
__device__ __forceinline__ void put_row16(T* __restrict__ dst, int left, const float* y)
{
    T t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = (T)y[i];
    if (left >= 16) {
        __builtin_memcpy(dst, t, sizeof t);
    } else {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < left) dst[i] = t[i];
    }
}

// the sum over the LANES neighbouring lanes of a row: the neighbour, the other pair, the other half of eight, of sixteen, and so on
template <int LANES>
__device__ __forceinline__ double over_lanes(double x)
{
    auto dpp = [](double v, auto ctrl) {
        return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(v), decltype(ctrl)::value, 0xf, 0xf, true),
                                __builtin_amdgcn_mov_dpp(__double2loint(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    x += dpp(x, std::integral_constant<int, 0xB1>());
    x += dpp(x, std::integral_constant<int, 0x4E>());
    x += dpp(x, std::integral_constant<int, 0x141>());
    if constexpr (LANES > 8) x += dpp(x, std::integral_constant<int, 0x140>());
    if constexpr (LANES > 16) x += __shfl_xor(x, 16);
    if constexpr (LANES > 32) x += __shfl_xor(x, 32);
    return x;
}

// A row has LANES lanes, or with LANES 64 `waves` wavefronts of a workgroup, each with 16 columns a lane and piece.  (bf16 with a residual: 8192 x 8192
// 102 us, 4.6 TB/s; 16384 x 2048 43 us, 5.4 TB/s, partly in the last-level cache; 32768 x 96 7 us.)
template <class T, class W, int FORMAT, int LANES, int PIECES>
__global__ __launch_bounds__(512) void rms_norm_kernel(NormView g, int waves)
{
    const int lane = threadIdx.x & (LANES - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __shared__ double part[8];
    const int64_t row = waves == 1 ? (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES : blockIdx.x;
    if (row >= g.out.rows) return;                           // (only where rows do not meet in LDS)
    const int cols = g.out.cols, col0 = (waves == 1 ? 0 : wave) * 1024 + 16 * lane, step = waves * 1024;
    const T *x = static_cast<const T*>(g.x) + row * g.x_ld, *r = static_cast<const T*>(g.residual) + row * g.residual_ld;
    T tx[PIECES][16], tr[PIECES][16];
    W tw[PIECES][16];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) get16(x + col0 + p * step, cols - col0 - p * step, tx[p]);
    if (g.residual) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) get16(r + col0 + p * step, cols - col0 - p * step, tr[p]);
    }
    if (g.weight) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) get16(static_cast<const W*>(g.weight) + col0 + p * step, cols - col0 - p * step, tw[p]);
    }
    float s[PIECES][16];
    double squares = 0.0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[p][i] = g.residual ? (float)tx[p][i] + (float)tr[p][i] : (float)tx[p][i];
            squares = fma((double)s[p][i], (double)s[p][i], squares);
        }
    if (g.sum) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) put_row16(static_cast<T*>(g.sum) + row * g.sum_ld + col0 + p * step, cols - col0 - p * step, s[p]);
    }
    squares = over_lanes<LANES>(squares);
    if (LANES == 64 && waves > 1) {
        if (lane == 0) part[wave] = squares;
        __syncthreads();
        squares = part[0];
        for (int w = 1; w < waves; ++w) squares += part[w];
    }
    // 1 / rms = by 2^power, by in [1, 2]: the row takes the power, which rounds nothing, and `by`, common to all values of a block, goes into its scale.
    const double mean = squares / cols + (double)g.eps, inv = mean > 0.0 ? 1.0 / sqrt(mean) : 0.0;
    const bool fine = mean - mean == 0.0;                                 // else an Inf or NaN in the row: NaN throughout
    const int power = fine ? __builtin_amdgcn_frexp_exp(inv) - 1 : 0;
    const float by = fine ? (float)ldexp(inv, -power) : __builtin_nanf("");
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int col = col0 + p * step, left = cols - col;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[p][i] = __builtin_amdgcn_ldexpf(s[p][i], power);
            if (g.weight) s[p][i] *= (float)tw[p][i];
        }
        const float scale = put16_by<FORMAT>(g.out.values + row * g.out.ld + col, left, most_of_8(most16(s[p])), s[p], by);
        if ((lane & 7) == 0 && left > 0) g.out.scales[(int64_t)(col / 128) * g.out.ld_scales + row] = scale;
        if (g.norm) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[p][i] *= by;
            put_row16(static_cast<T*>(g.norm) + row * g.norm_ld + col, left, s[p]);
        }
    }
}

// silu(gate) * up = gate up / (1 + exp(-gate)); exp(-gate) is kept between 2^-145 and 2^127.97, whose reciprocal below 2^-126 the instruction makes 0, so that gates of
// any size to that side give 0.  exp(-gate) = 2^t 2^rest: t is the product with log2(e) rounded to
// fp32, rest what that leaves out (with t alone the result is off by |gate| units, and more values fall to the other side of an 8-bit border).  The
// reciprocal is corrected once.
__device__ __forceinline__ float swiglu(float gate, float up)
{
    const float x = __builtin_amdgcn_fmed3f(gate, -88.7f, 100.f);           // (what is not finite comes back with the last products)
    const float t = -1.44269504f * x, rest = fmaf(-1.92596299e-8f, x, fmaf(-1.44269504f, x, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = fmaf(e, 0.693147181f * rest, e);
    const float d = 1.f + e;
    float r = __builtin_amdgcn_rcpf(d);
    r = fmaf(fmaf(-d, r, 1.f), r, r);
    return gate * r * up;
}

// Eight lanes have a block, whichever row it is in.  (bf16, 32768 x 2048: 69 to 73 us, 4.6 to 4.9 TB/s; fp32 113, 5.3; with 36 instructions a value instead of 25 it was bound by them, 92.)
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void swiglu_kernel(const T* __restrict__ x, int64_t ld, Fp8View out)
{
    const int lane = threadIdx.x & 7;
    const Item at = item_of((int64_t)blockIdx.x * 32, threadIdx.x >> 3, (out.cols + 127) / 128);
    const int64_t row = at.row;
    const int col = at.piece * 128 + 16 * lane, left = out.cols - col;
    if (row >= out.rows) return;
    T gate[16], up[16];
    get16(x + row * ld + col, left, gate);
    get16(x + row * ld + out.cols + col, left, up);
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = swiglu((float)gate[i], (float)up[i]);
    const float scale = put16_by<FORMAT>(out.values + row * out.ld + col, left, most_of_8(most16(y)), y);
    if (lane == 0) out.scales[(int64_t)at.piece * out.ld_scales + row] = scale;
}

template <class T, class W, int FORMAT>
static hipError_t norm_of(hipStream_t s, const NormView& g)
{
    const int cols = g.out.cols;
    auto rows_of = [&](int lanes) { return dim3((unsigned)((g.out.rows + 256 / lanes - 1) / (256 / lanes))); };
    if (cols <= 128) hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 8, 1>), rows_of(8), dim3(256), 0, s, g, 1);
    else if (cols <= 256) hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 16, 1>), rows_of(16), dim3(256), 0, s, g, 1);
    else if (cols <= 512) hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 32, 1>), rows_of(32), dim3(256), 0, s, g, 1);
    else if (cols <= 1024) hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 64, 1>), rows_of(64), dim3(256), 0, s, g, 1);
    else {
        // up to 8 wavefronts, which is what shares a row best (8192 x 8192: 8 with a piece each 102 us, 4 with two 107, 2 with four 133)
        const int pieces = cols <= 8192 ? 1 : cols <= 16384 ? 2 : 4, waves = (cols + 1024 * pieces - 1) / (1024 * pieces);
        const dim3 grid((unsigned)g.out.rows), block(64 * waves);
        if (pieces == 1) hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 64, 1>), grid, block, 0, s, g, waves);
        else if (pieces == 2) hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 64, 2>), grid, block, 0, s, g, waves);
        else hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 64, 4>), grid, block, 0, s, g, waves);
    }
    return hipGetLastError();
}

template <class T>
static hipError_t norm_of(hipStream_t s, const NormView& g, int weight_type)
{
    const bool e4 = g.out.format == FOBQ_E4M3;
    if (weight_type == FOBQ_F32) return e4 ? norm_of<T, float, FOBQ_E4M3>(s, g) : norm_of<T, float, FOBQ_E5M2>(s, g);
    return e4 ? norm_of<T, T, FOBQ_E4M3>(s, g) : norm_of<T, T, FOBQ_E5M2>(s, g);
}

hipError_t launch_rms_norm(hipStream_t s, const NormView& g, int type, int weight_type)
{
    if (type == FOBQ_F32) return norm_of<float>(s, g, FOBQ_F32);
    return type == FOBQ_BF16 ? norm_of<bf16_t>(s, g, weight_type) : norm_of<f16_t>(s, g, weight_type);
}

template <class T>
static hipError_t swiglu_of(hipStream_t s, const void* x, int64_t ld, const Fp8View& out)
{
    const int64_t blocks = (int64_t)out.rows * ((out.cols + 127) / 128);
    const dim3 grid((unsigned)((blocks + 31) / 32)), block(256);
    const T* t = static_cast<const T*>(x);
    if (out.format == FOBQ_E4M3) hipLaunchKernelGGL((swiglu_kernel<T, FOBQ_E4M3>), grid, block, 0, s, t, ld, out);
    else hipLaunchKernelGGL((swiglu_kernel<T, FOBQ_E5M2>), grid, block, 0, s, t, ld, out);
    return hipGetLastError();
}

hipError_t launch_swiglu(hipStream_t s, const void* x, int type, int64_t ld, const Fp8View& out)
{
    if (type == FOBQ_F32) return swiglu_of<float>(s, x, ld, out);
    return type == FOBQ_BF16 ? swiglu_of<bf16_t>(s, x, ld, out) : swiglu_of<f16_t>(s, x, ld, out);
}

}  // namespace fobq
