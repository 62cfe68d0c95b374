// C ABI of the calls that run a quantized network: argument checks and launches.  They allocate nothing and wait for nothing.
#include "api_lowbit.h"
#include "kv4.h"

#include <algorithm>

namespace fobq {

int check_matrix(fobq_ctx* ctx, const fobq_fp8_matrix* m, const char* name, Fp8View* v)
{
    if (!m) return set_err(ctx, FOBQ_EINVAL, "%s is NULL", name);
    if (m->rows < 0 || m->rows >= MAX_SIDE || m->cols < 0 || m->cols >= MAX_SIDE)
        return set_err(ctx, FOBQ_EINVAL, "%s: rows and cols must be in 0..%lld", name, (long long)MAX_SIDE - 1);
    if (m->rows * std::max<int64_t>(1, (m->cols + 511) / 512) > MAX_ROWS)       // (no columns: a product's results are written all the same)
        return set_err(ctx, FOBQ_EINVAL, "%s: rows times 512 columns must be no more than %lld (got %lld x %lld)", name, (long long)MAX_ROWS, (long long)m->rows, (long long)m->cols);
    if (m->format != FOBQ_E4M3 && m->format != FOBQ_E5M2) return set_err(ctx, FOBQ_EINVAL, "%s: unknown format %d", name, m->format);
    if (m->rows_per_scale != 1 && m->rows_per_scale != 128)
        return set_err(ctx, FOBQ_EINVAL, "%s: rows_per_scale must be 1 or 128 (got %d)", name, m->rows_per_scale);
    if (m->ld < m->cols || m->ld % 16 != 0)
        return set_err(ctx, FOBQ_EINVAL, "%s: ld (%lld) must be a multiple of 16 and no less than cols", name, (long long)m->ld);
    if (m->ld_scales < (m->rows + m->rows_per_scale - 1) / m->rows_per_scale)
        return set_err(ctx, FOBQ_EINVAL, "%s: ld_scales (%lld) is less than the blocks of a column", name, (long long)m->ld_scales);
    if (m->rows > 0 && m->cols > 0) {
        if (!m->values || !m->scales) return set_err(ctx, FOBQ_EINVAL, "%s: values or scales is NULL", name);
        if (!aligned(m->values, 16) || !aligned(m->scales, 4)) return set_err(ctx, FOBQ_EINVAL, "%s: values must be 16-byte aligned, scales 4-byte", name);
    }
    *v = Fp8View{static_cast<uint8_t*>(m->values), m->scales, (int)m->rows, (int)m->cols, m->ld, m->ld_scales, m->rows_per_scale, m->format};
    return FOBQ_OK;
}

static int check_kv4(fobq_ctx* ctx, const fobq_kv4_cache* c, const fobq_kv4_batch* b, Kv4View* cv, Kv4Seqs* sv)
{
    if (!c || !b) return set_err(ctx, FOBQ_EINVAL, "cache or batch is NULL");
    if (c->reserved != 0) return set_err(ctx, FOBQ_EINVAL, "reserved must be 0");
    if (c->pages < 1 || c->pages > INT32_MAX) return set_err(ctx, FOBQ_EINVAL, "pages must be in 1..2^31 - 1 (got %lld)", (long long)c->pages);
    if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
        return set_err(ctx, FOBQ_EINVAL, "page_size must be a power of two in 16..4096 (got %d)", c->page_size);
    if (c->heads < 1 || c->heads > 1024) return set_err(ctx, FOBQ_EINVAL, "heads must be in 1..1024 (got %d)", c->heads);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        return set_err(ctx, FOBQ_EINVAL, "head_dim must be 64, 128 or 256 (got %d)", c->head_dim);
    if (!c->k_codes || !c->v_codes || !c->k_grids || !c->v_grids) return set_err(ctx, FOBQ_EINVAL, "a part of the cache is NULL");
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_grids, 16) || !aligned(c->v_grids, 16))
        return set_err(ctx, FOBQ_EINVAL, "the parts of the cache must be 16-byte aligned");
    if (b->rows < 0 || b->rows > MAX_ROWS) return set_err(ctx, FOBQ_EINVAL, "rows must be in 0..%lld (got %lld)", (long long)MAX_ROWS, (long long)b->rows);
    if (b->n_seqs < 0 || b->n_seqs > (1 << 20)) return set_err(ctx, FOBQ_EINVAL, "n_seqs must be in 0..2^20 (got %d)", b->n_seqs);
    int shift = 4;
    while ((1 << shift) < c->page_size) ++shift;
    if (b->max_pages < 0 || b->table_ld < b->max_pages || ((int64_t)b->max_pages << shift) >= ((int64_t)1 << 30))
        return set_err(ctx, FOBQ_EINVAL, "max_pages (%d) must be in 0..table_ld, and max_pages * page_size below 2^30", b->max_pages);
    if (b->n_seqs > 0 && b->rows > 0 && (!b->lengths || (b->max_pages > 0 && !b->table))) return set_err(ctx, FOBQ_EINVAL, "table or lengths is NULL");
    *cv = Kv4View{c->k_codes, c->v_codes, c->k_grids, c->v_grids, (int)c->pages, c->heads, c->head_dim, shift};
    *sv = Kv4Seqs{b->table, b->lengths, b->starts, b->table_ld, b->n_seqs, b->max_pages, (int)b->rows};
    return FOBQ_OK;
}

static int check_attention(fobq_ctx* ctx, const fobq_kv4_cache* c, const fobq_kv4_batch* b, const fobq_kv4_query* q, Kv4View* cv, Kv4Seqs* sv, Kv4Plan* p)
{
    int rc = check_kv4(ctx, c, b, cv, sv);
    if (rc) return rc;
    if (!q) return set_err(ctx, FOBQ_EINVAL, "query is NULL");
    if (q->reserved != 0) return set_err(ctx, FOBQ_EINVAL, "reserved must be 0");
    if (q->type != FOBQ_BF16 && q->type != FOBQ_F16) return set_err(ctx, FOBQ_EINVAL, "queries must be BF16 or F16 (got type %d)", q->type);
    if (q->group < 1 || q->group > 1024) return set_err(ctx, FOBQ_EINVAL, "group must be in 1..1024 (got %d)", q->group);
    if (b->rows * q->group * c->heads >= MAX_SIDE) return set_err(ctx, FOBQ_EINVAL, "rows * query heads must be below %lld", (long long)MAX_SIDE);
    if (q->window < 0) return set_err(ctx, FOBQ_EINVAL, "window must be >= 0 (got %d)", q->window);
    if (q->max_length < 0) return set_err(ctx, FOBQ_EINVAL, "max_length must be >= 0");
    if (!(q->scale - q->scale == 0.f)) return set_err(ctx, FOBQ_EINVAL, "scale must be finite");
    if (q->q_row < 0 || q->q_head < 0 || q->out_row < 0 || q->out_head < 0) return set_err(ctx, FOBQ_EINVAL, "strides must be >= 0");
    const int64_t holds = (int64_t)b->max_pages << cv->shift;
    int64_t longest = q->max_length > 0 && q->max_length < holds ? q->max_length : holds;
    if (q->window > 0) longest = longest < q->window ? longest : q->window;
    *p = kv4_attention_plan(ctx->cus, cv->dim, cv->heads, q->group, sv->n_seqs, sv->rows, longest);
    if (p->tiles * cv->heads > MAX_TILES)
        return set_err(ctx, FOBQ_EINVAL, "rows * query heads / %d + n_seqs * heads must be no more than %lld", p->tile, (long long)MAX_TILES);
    return FOBQ_OK;
}

int lowbit_debug_plan(int32_t what, const int64_t* in, int32_t n_in, int64_t* out, int32_t n_out)
{
    if (what == FOBQ_PLAN_FP8_MATMUL && n_in == 6 && n_out == 5) {
        for (int i = 0; i < 4; ++i)
            if (in[i] < (i ? 0 : 16) || in[i] >= (i ? MAX_SIDE : 4096)) return FOBQ_EINVAL;
        if (!is_float((int)in[4]) || (in[5] != 1 && in[5] != 128)) return FOBQ_EINVAL;
        const Fp8Plan p = fp8_matmul_plan((int)in[0], in[1], in[2], in[3], (int)in[4], (int)in[5]);
        out[0] = p.tm; out[1] = p.tn; out[2] = p.parts; out[3] = p.blocks_per_part; out[4] = fp8_matmul_workspace(p, in[1], in[2]);
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_KV4_ATTENTION && n_in == 7 && n_out == 5) {
        if (in[0] < 16 || in[0] > 4096 || (in[1] != 64 && in[1] != 128 && in[1] != 256) || in[2] < 1 || in[2] > 1024 || in[3] < 1 || in[3] > 1024 || in[4] < 1 ||
            in[4] > (1 << 20) || in[5] < 0 || in[5] * in[2] * in[3] >= MAX_SIDE || in[6] < 0 || in[6] >= ((int64_t)1 << 30)) return FOBQ_EINVAL;
        const Kv4Plan p = kv4_attention_plan((int)in[0], (int)in[1], (int)in[2], (int)in[3], (int)in[4], in[5], in[6]);
        out[0] = p.tile; out[1] = p.share; out[2] = p.slots; out[3] = p.tiles; out[4] = kv4_attention_workspace(p, (int)in[1], (int)in[2]);
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_KV4_PLACE && n_in >= 6 && n_out == 3) {
        const int64_t n = in[3], width = in[2];
        if (n < 1 || n > 64 || width < 0 || width > 64 || n_in != 6 + n + n + 1 + n * width) return FOBQ_EINVAL;
        if (in[0] < 16 || in[0] > 4096 || (in[0] & (in[0] - 1)) || in[1] < 1 || in[1] > INT32_MAX || in[4] < 0 || in[4] > MAX_ROWS || in[5] < 0 ||
            in[5] > MAX_ROWS) return FOBQ_EINVAL;
        int32_t lengths[64], starts[65], table[64 * 64];
        for (int i = 0; i < n; ++i) lengths[i] = (int32_t)in[6 + i];
        for (int i = 0; i <= n; ++i) starts[i] = (int32_t)in[6 + n + i];
        for (int i = 0; i < n * width; ++i) table[i] = (int32_t)in[6 + 2 * n + 1 + i];
        int shift = 0;
        while ((1ll << shift) < in[0]) ++shift;
        const Kv4Seqs s{table, lengths, starts, width, (int)n, (int)width, (int)in[4]};
        int b = 0;                                          // as the wavefronts search: the last sequence that begins at or before the row
        for (int i = 1; i < n; ++i)
            if (kv4_rows(starts, i, s.rows).first <= in[5]) b = i;
        const Kv4Place p = kv4_place(s, (int)in[1], shift, b, (int)in[5]);
        out[0] = b; out[1] = p.page; out[2] = p.place;
        return FOBQ_OK;
    }
    auto address = [](int64_t x) { return reinterpret_cast<void*>(static_cast<uintptr_t>(x)); };
    if (what == FOBQ_PLAN_FP8_CHECK && n_in == 8 && n_out == 1) {
        const fobq_fp8_matrix m{address(in[6]), static_cast<float*>(address(in[7])), in[0], in[1], in[2], in[3], (int32_t)in[4], (int32_t)in[5]};
        Fp8View v;
        out[0] = check_matrix(nullptr, &m, "matrix", &v);
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_KV4_CHECK && n_in == 15 && n_out == 1) {
        const fobq_kv4_cache c{static_cast<uint8_t*>(address(in[9])), static_cast<uint8_t*>(address(in[10])), static_cast<uint32_t*>(address(in[11])),
                               static_cast<uint32_t*>(address(in[12])), in[0], (int32_t)in[1], (int32_t)in[2], (int32_t)in[3], (int32_t)in[4]};
        const fobq_kv4_batch b{static_cast<int32_t*>(address(in[13])), static_cast<int32_t*>(address(in[14])), nullptr, in[6], in[8], (int32_t)in[5], (int32_t)in[7]};
        Kv4View cv;
        Kv4Seqs sv;
        out[0] = check_kv4(nullptr, &c, &b, &cv, &sv);
        return FOBQ_OK;
    }
    return experts_debug_plan(what, in, n_in, out, n_out);
}

}  // namespace fobq

using namespace fobq;

extern "C" {

int fobq_fp8_quantize(fobq_ctx* ctx, const void* X, int32_t type, int64_t ld, const fobq_fp8_matrix* out)
{
    if (!ctx) return FOBQ_EINVAL;
    Fp8View v;
    int rc = check_matrix(ctx, out, "out", &v);
    if (rc) return rc;
    if (!is_float(type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", type);
    if (ld < out->cols) return set_err(ctx, FOBQ_EINVAL, "ld (%lld) is less than cols", (long long)ld);
    if (out->rows == 0 || out->cols == 0) return FOBQ_OK;
    if (!X || !aligned(X, float_size(type))) return set_err(ctx, FOBQ_EINVAL, "X is NULL or not aligned to its elements");
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_fp8_quantize(ctx->stream, X, type, ld, v), "quantize to 8-bit blocks");
    return FOBQ_OK;
}

int fobq_fp8_from_codes(fobq_ctx* ctx, const uint8_t* codes, const float* scales, const float* zeros, int32_t bits, int32_t group, const fobq_fp8_matrix* out)
{
    if (!ctx) return FOBQ_EINVAL;
    Fp8View v;
    int rc = check_matrix(ctx, out, "out", &v);
    if (rc) return rc;
    if (bits < 2 || bits > 4) return set_err(ctx, FOBQ_EINVAL, "codes of 2..4 bits are exact in e4m3 (got %d)", bits);
    if (out->format != FOBQ_E4M3 || out->rows_per_scale != 1) return set_err(ctx, FOBQ_EINVAL, "out must be e4m3 with a scale per row");
    if (group < 0 || group % 128 != 0 || (group > 0 && out->cols % group != 0))
        return set_err(ctx, FOBQ_EINVAL, "group (%d) must be 0 or a multiple of 128 that divides the columns", group);
    if (out->rows == 0 || out->cols == 0) return FOBQ_OK;
    if (!codes || !scales || !zeros) return set_err(ctx, FOBQ_EINVAL, "codes, scales or zeros is NULL");
    if (!aligned(scales, 4) || !aligned(zeros, 4)) return set_err(ctx, FOBQ_EINVAL, "scales and zeros must be 4-byte aligned");
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_fp8_from_codes(ctx->stream, codes, scales, zeros, group, v), "codes to 8-bit blocks");
    return FOBQ_OK;
}

int fobq_fp8_matmul_workspace(fobq_ctx* ctx, int64_t m, int64_t n, int64_t k, int32_t type, int64_t* bytes)
{
    if (!ctx) return FOBQ_EINVAL;
    if (!bytes || m < 0 || n < 0 || k < 0 || m >= MAX_SIDE || n >= MAX_SIDE || k >= MAX_SIDE)
        return set_err(ctx, FOBQ_EINVAL, "bytes is NULL, or a size is not in 0..%lld", (long long)MAX_SIDE - 1);
    if (!is_float(type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", type);
    *bytes = fp8_matmul_workspace(fp8_matmul_plan(ctx->cus, m, n, k, type, 128), m, n);
    return FOBQ_OK;
}

int fobq_fp8_matmul(fobq_ctx* ctx, const fobq_fp8_matrix* A, const fobq_fp8_matrix* B, void* Y, int32_t type, int64_t ld, void* work, int64_t work_bytes)
{
    if (!ctx) return FOBQ_EINVAL;
    Fp8View a, b;
    int rc = check_matrix(ctx, A, "A", &a);
    if (!rc) rc = check_matrix(ctx, B, "B", &b);
    if (rc) return rc;
    if (a.per != 1) return set_err(ctx, FOBQ_EINVAL, "A must have a scale per row");
    if (a.cols != b.cols) return set_err(ctx, FOBQ_EINVAL, "A has %d columns, B %d", a.cols, b.cols);
    if (a.ld >= MAX_APART || b.ld >= MAX_APART)
        return set_err(ctx, FOBQ_EINVAL, "rows must be less than %lld bytes apart", (long long)MAX_APART);
    if (!is_float(type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", type);
    if (ld < b.rows) return set_err(ctx, FOBQ_EINVAL, "ld (%lld) is less than the rows of B", (long long)ld);
    if (((int64_t)a.rows + 63) / 64 * (((int64_t)b.rows + 63) / 64) > MAX_TILES)
        return set_err(ctx, FOBQ_EINVAL, "Y has more than %lld tiles of 64 x 64", (long long)MAX_TILES);
    if (a.rows == 0 || b.rows == 0) return FOBQ_OK;
    if (!Y || !aligned(Y, float_size(type))) return set_err(ctx, FOBQ_EINVAL, "Y is NULL or not aligned to its elements");
    const Fp8Plan p = fp8_matmul_plan(ctx->cus, a.rows, b.rows, a.cols, type, b.per);
    const int64_t need = fp8_matmul_workspace(p, a.rows, b.rows);
    if (work_bytes < need || (need > 0 && (!work || !aligned(work, 16))))
        return set_err(ctx, FOBQ_EINVAL, "work must be %lld bytes, 16-byte aligned (got %lld)", (long long)need, (long long)work_bytes);
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_fp8_matmul(ctx->stream, p, a, b, Y, type, ld, need ? static_cast<float*>(work) : nullptr), "product of 8-bit blocks");
    return FOBQ_OK;
}

static int check_rows(fobq_ctx* ctx, int type, const void* K, int64_t k_row, int64_t k_head, const void* V, int64_t v_row, int64_t v_head)
{
    if (!K || !V || !aligned(K, float_size(type)) || !aligned(V, float_size(type)))
        return set_err(ctx, FOBQ_EINVAL, "K or V is NULL or not aligned to its elements");
    if (k_row < 0 || k_head < 0 || v_row < 0 || v_head < 0) return set_err(ctx, FOBQ_EINVAL, "strides must be >= 0");
    return FOBQ_OK;
}

int fobq_kv4_append(fobq_ctx* ctx, const fobq_kv4_cache* cache, const fobq_kv4_batch* batch, int32_t type, const void* K, int64_t k_row, int64_t k_head,
                    const void* V, int64_t v_row, int64_t v_head)
{
    if (!ctx) return FOBQ_EINVAL;
    Kv4View c;
    Kv4Seqs s;
    int rc = check_kv4(ctx, cache, batch, &c, &s);
    if (rc) return rc;
    if (type != FOBQ_BF16 && type != FOBQ_F16) return set_err(ctx, FOBQ_EINVAL, "keys and values must be BF16 or F16 (got type %d)", type);
    if (s.rows == 0 || s.n_seqs == 0) return FOBQ_OK;
    if ((rc = check_rows(ctx, type, K, k_row, k_head, V, v_row, v_head))) return rc;
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_kv4_append(ctx->stream, c, s, type, K, k_row, k_head, V, v_row, v_head), "append to the cache");
    return FOBQ_OK;
}

int fobq_kv4_read(fobq_ctx* ctx, const fobq_kv4_cache* cache, const fobq_kv4_batch* batch, int32_t type, void* K, int64_t k_row, int64_t k_head, void* V,
                  int64_t v_row, int64_t v_head)
{
    if (!ctx) return FOBQ_EINVAL;
    Kv4View c;
    Kv4Seqs s;
    int rc = check_kv4(ctx, cache, batch, &c, &s);
    if (rc) return rc;
    if (!is_float(type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", type);
    if (s.rows == 0 || s.n_seqs == 0) return FOBQ_OK;
    if ((rc = check_rows(ctx, type, K, k_row, k_head, V, v_row, v_head))) return rc;
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_kv4_read(ctx->stream, c, s, type, K, k_row, k_head, V, v_row, v_head), "read the cache");
    return FOBQ_OK;
}

int fobq_kv4_attention_workspace(fobq_ctx* ctx, const fobq_kv4_cache* cache, const fobq_kv4_batch* batch, const fobq_kv4_query* query, int64_t* bytes)
{
    if (!ctx) return FOBQ_EINVAL;
    if (!bytes) return set_err(ctx, FOBQ_EINVAL, "bytes is NULL");
    Kv4View c;
    Kv4Seqs s;
    Kv4Plan p;
    const int rc = check_attention(ctx, cache, batch, query, &c, &s, &p);
    if (rc) return rc;
    *bytes = kv4_attention_workspace(p, c.dim, c.heads);
    return FOBQ_OK;
}

int fobq_kv4_attention(fobq_ctx* ctx, const fobq_kv4_cache* cache, const fobq_kv4_batch* batch, const fobq_kv4_query* query, void* work, int64_t work_bytes)
{
    if (!ctx) return FOBQ_EINVAL;
    Kv4View c;
    Kv4Seqs s;
    Kv4Plan p;
    int rc = check_attention(ctx, cache, batch, query, &c, &s, &p);
    if (rc) return rc;
    if (s.rows == 0 || s.n_seqs == 0) return FOBQ_OK;
    if (!query->Q || !query->out || !aligned(query->Q, 2) || !aligned(query->out, 2) || !aligned(query->lse, 4))
        return set_err(ctx, FOBQ_EINVAL, "Q or out is NULL, or Q, out or lse is not aligned to its elements");
    const int64_t need = kv4_attention_workspace(p, c.dim, c.heads);
    if (work_bytes < need || (need > 0 && (!work || !aligned(work, 16))))
        return set_err(ctx, FOBQ_EINVAL, "work must be %lld bytes, 16-byte aligned (got %lld)", (long long)need, (long long)work_bytes);
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    const Kv4Query q{query->Q, query->q_row, query->q_head, query->out, query->out_row, query->out_head, query->lse,
                     query->group, query->causal, query->window, query->scale};
    FOBQ_TRY(launch_kv4_attention(ctx->stream, p, c, s, query->type, q, need ? static_cast<float*>(work) : nullptr), "attention over the cache");
    return FOBQ_OK;
}

}  // extern "C"
