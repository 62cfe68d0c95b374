// What stands in front of and between products of 8-bit blocks: the residual's addition with a root-mean-square norm, and the gated
// activation, both straight into blocks of 128 columns with a scale per row.
//
// Memory bound: a lane has 16 columns of a row, eight lanes a block, and everything between the loads and the 8-bit values stays in
// registers.  The sum of squares is in fp64, which no row of finite values passes, and 1 / rms enters as a power of two, exact, and a factor
// between 1/2 and 2, so that rows of very large and very small values lose nothing either.  Both cost a few instructions that memory hides.
#include "fp8.h"

namespace fobq {

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

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    return x;
}

// A row has `waves` wavefronts of a workgroup, 1024 columns each and PIECES times that; with one, a workgroup has four rows.
template <class T, class W, int FORMAT, int PIECES>
__global__ __launch_bounds__(1024) void rms_norm_kernel(NormView g, int waves)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __shared__ double part[16];
    const int64_t row = waves == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (row >= g.out.rows) return;                           // (only where every wavefront has a row of its own)
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
    squares = wave_sum(squares);
    if (waves > 1) {
        if (lane == 0) part[wave] = squares;
        __syncthreads();
        squares = part[0];
        for (int w = 1; w < waves; ++w) squares += part[w];
    }
    const double mean = squares / cols + (double)g.eps;
    // s / rms = (s * pre) * inv, pre a power of two
    float pre = 0.f, inv = 0.f;
    if (mean > 0.0) {
        const double rms = sqrt(mean);
        const int e = min(126, max(-126, -ilogb(rms)));
        pre = ldexpf(1.f, e);
        inv = (float)(1.0 / (rms * ldexp(1.0, e)));
    }
    if (!(mean - mean == 0.0)) inv = __builtin_nanf("");     // an Inf or NaN in the row
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int col = col0 + p * step, left = cols - col;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[p][i] = s[p][i] * pre * inv;
            if (g.weight) s[p][i] *= (float)tw[p][i];
        }
        const Fp8Scale b = fp8_scale<FORMAT>(most_of_8(most16(s[p])));
        put16<float, FORMAT>(g.out.values + row * g.out.ld + col, left, b, s[p]);
        if ((lane & 7) == 0 && left > 0) g.out.scales[(int64_t)(col / 128) * g.out.ld_scales + row] = b.scale;
        if (g.norm) put_row16(static_cast<T*>(g.norm) + row * g.norm_ld + col, left, s[p]);
    }
}

// silu(gate) * up.  Where exp(g) falls below 2^-126 it counts as 0; what is not finite is NaN.
__device__ __forceinline__ float swiglu(float gate, float up)
{
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(gate)), r = 1.f / (1.f + e);
    return gate * (gate < 0.f ? e * r : r) * up;
}

template <class T, int FORMAT>
__global__ __launch_bounds__(256) void swiglu_kernel(const T* __restrict__ x, int64_t ld, Fp8View out)
{
    const int lane = threadIdx.x & 63;
    const Item at = item_of((int64_t)blockIdx.x * 4, threadIdx.x >> 6, (out.cols + 1023) / 1024);
    const int64_t row = at.row;
    const int col = at.piece * 1024 + 16 * lane, left = out.cols - col;
    if (row >= out.rows) return;
    T gate[16], up[16];
    get16(x + row * ld + col, left, gate);
    get16(x + row * ld + out.cols + col, left, up);
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = swiglu((float)gate[i], (float)up[i]);
    const Fp8Scale s = fp8_scale<FORMAT>(most_of_8(most16(y)));
    put16<float, FORMAT>(out.values + row * out.ld + col, left, s, y);
    if ((lane & 7) == 0 && left > 0) out.scales[(int64_t)(col / 128) * out.ld_scales + row] = s.scale;
}

template <class T, class W, int FORMAT>
static hipError_t norm_of(hipStream_t s, const NormView& g)
{
    const int pieces = g.out.cols <= 16384 ? 1 : 2, waves = (g.out.cols + 1024 * pieces - 1) / (1024 * pieces);
    const dim3 grid((unsigned)(waves == 1 ? (g.out.rows + 3) / 4 : g.out.rows)), block(waves == 1 ? 256 : 64 * waves);
    if (pieces == 1) hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 1>), grid, block, 0, s, g, waves);
    else hipLaunchKernelGGL((rms_norm_kernel<T, W, FORMAT, 2>), grid, block, 0, s, g, waves);
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
    const int64_t items = (int64_t)out.rows * ((out.cols + 1023) / 1024);
    const dim3 grid((unsigned)((items + 3) / 4)), block(256);
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
