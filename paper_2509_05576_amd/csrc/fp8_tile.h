// What the products of 8-bit blocks share: the matrix instructions on a block of 128 columns, copies of tiles straight into LDS and where
// their rows lie there.
#pragma once
#include "lowbit.h"

#ifdef __HIPCC__
namespace fobq {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));

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

// Waits until at most LEFT copies of this wavefront are under way, and for the whole workgroup to be there.  (A barrier of the language
// waits for all of them.)
template <int LEFT>
__device__ __forceinline__ void wait_and_meet()
{
    static_assert(LEFT < 64, "a count of six bits");
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

}  // namespace fobq
#endif
