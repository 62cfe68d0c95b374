// Matrices in 8-bit floating point with a scale for each block of 128 columns and 1 or 128 rows: from 16- and 32-bit matrices, and
// from the codes of a quantized layer.
//
// fp8.h has the scales and the rounding.
#include "fp8.h"

namespace fobq {

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
