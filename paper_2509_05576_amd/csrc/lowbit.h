// What the kernels on 16- and 8-bit data share: element types, 8 elements at a time, and the views that the C entry points make of
// their arguments.
#pragma once
#include "fobq_internal.h"

namespace fobq {

#ifdef __HIPCC__
typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// 8 elements that begin anywhere (global memory takes accesses of any alignment; an aligned one is as fast as if the type said so)
template <class T>
__device__ __forceinline__ void load8(const T* __restrict__ p, float* x)
{
    T t[8];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)t[i];
}
template <class T>
__device__ __forceinline__ void store8(T* __restrict__ p, const float* x)
{
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)x[i];
    __builtin_memcpy(p, t, sizeof t);
}
#endif

// a matrix of 8-bit values in blocks (fobq_fp8_matrix, checked)
struct Fp8View { uint8_t* values; float* scales; int rows, cols; int64_t ld, ld_scales; int per, format; };

hipError_t launch_fp8_quantize(hipStream_t s, const void* x, int type, int64_t ld, const Fp8View& out);
hipError_t launch_fp8_from_codes(hipStream_t s, const uint8_t* codes, const float* scales, const float* zeros, int group, const Fp8View& out);

// The product: tile edges and parts of the contraction (parts > 1: fp32 partial results in `work`, added by a second launch).
struct Fp8Plan { int tm, tn, parts; int64_t blocks_per_part; };
Fp8Plan fp8_matmul_plan(int cus, int64_t m, int64_t n, int64_t k, int type, int per);
int64_t fp8_matmul_workspace(const Fp8Plan& p, int64_t m, int64_t n);
hipError_t launch_fp8_matmul(hipStream_t s, const Fp8Plan& p, const Fp8View& a, const Fp8View& b, void* y, int type, int64_t ldy, float* work);

// the cache and the sequences of a call (fobq_kv4_cache, fobq_kv4_batch, checked); a page has 1 << shift tokens
struct Kv4View { uint8_t *k_codes, *v_codes; uint32_t *k_grids, *v_grids; int pages, heads, dim, shift; };
struct Kv4Seqs { const int32_t *table, *lengths, *starts; int64_t table_ld; int n_seqs, max_pages, rows; };

hipError_t launch_kv4_append(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, int type, const void* k, int64_t k_row, int64_t k_head, const void* v,
                             int64_t v_row, int64_t v_head);
hipError_t launch_kv4_read(hipStream_t st, const Kv4View& c, const Kv4Seqs& s, int type, void* k, int64_t k_row, int64_t k_head, void* v, int64_t v_row,
                           int64_t v_head);

// Attention: query rows per workgroup (the rows of a sequence are its tokens times the query heads of a kv head), whether the
// wavefronts of a workgroup share them and go through the tokens in turn; tiles: workgroups of a head that hold all rows.  slots: 0, or the
// workgroups of a head where sequences are split into parts of equal size (partial results in `work`, joined by a second launch).
struct Kv4Plan { int tile, share, slots; int64_t tiles; };
Kv4Plan kv4_attention_plan(int cus, int dim, int heads, int group, int n_seqs, int64_t rows, int64_t longest);
int64_t kv4_attention_workspace(const Kv4Plan& p, int dim, int heads);
struct Kv4Query {
    const void* q; int64_t q_row, q_head; void* out; int64_t out_row, out_head; float* lse;
    int group, causal, window; float scale;
};
hipError_t launch_kv4_attention(hipStream_t st, const Kv4Plan& p, const Kv4View& c, const Kv4Seqs& s, int type, const Kv4Query& q, float* work);

}  // namespace fobq
