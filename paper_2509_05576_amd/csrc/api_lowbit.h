// What the C entry points of the calls that run a quantized network check and share.
#pragma once
#include "lowbit.h"

namespace fobq {

constexpr int64_t MAX_SIDE = (int64_t)1 << 29;      // rows and columns of a matrix, rows times query heads: products with 4 stay in 32 bits
// A launch has fewer than 2^32 threads: a wavefront for each row of the cache, or for 512 columns of a matrix's row; 256 for a tile.
constexpr int64_t MAX_ROWS = ((int64_t)1 << 26) - 4, MAX_TILES = ((int64_t)1 << 24) - 1;
constexpr int64_t MAX_APART = (int64_t)1 << 24;     // rows of a product's matrices: 256 of them stay within 32-bit offsets

inline int enter(fobq_ctx* ctx, const DeviceGuard& g) { return g.ok ? FOBQ_OK : set_err(ctx, FOBQ_EHIP, "cannot select device %d", ctx->device); }

inline bool aligned(const void* p, int to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

inline int float_size(int type) { return type == FOBQ_F32 ? 4 : 2; }
inline bool is_float(int type) { return type == FOBQ_F32 || type == FOBQ_BF16 || type == FOBQ_F16; }

int check_matrix(fobq_ctx* ctx, const fobq_fp8_matrix* m, const char* name, Fp8View* v);
int experts_debug_plan(int32_t what, const int64_t* in, int32_t n_in, int64_t* out, int32_t n_out);

}  // namespace fobq
