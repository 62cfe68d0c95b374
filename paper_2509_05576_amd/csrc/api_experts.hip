// C ABI of a feed-forward part of experts: argument checks and launches.  The calls allocate nothing and wait for nothing.
#include "api_lowbit.h"

#include <algorithm>

namespace fobq {

constexpr int MAX_EXPERTS = 1024, MAX_TOP = 32, MAX_GROUPS = 64, MAX_NORM_COLS = 32768;

static bool finite(float x) { return x - x == 0.f; }

static int check_norm(fobq_ctx* ctx, const fobq_norm* n, const fobq_fp8_matrix* out, NormView* v)
{
    Fp8View m;
    int rc = check_matrix(ctx, out, "out", &m);
    if (rc) return rc;
    if (!n) return set_err(ctx, FOBQ_EINVAL, "norm is NULL");
    if (n->reserved != 0) return set_err(ctx, FOBQ_EINVAL, "reserved must be 0");
    if (m.per != 1) return set_err(ctx, FOBQ_EINVAL, "out must have a scale per row");
    if (m.cols < 1 || m.cols > MAX_NORM_COLS) return set_err(ctx, FOBQ_EINVAL, "cols must be in 1..%d (got %d)", MAX_NORM_COLS, m.cols);
    if (!is_float(n->type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", n->type);
    if (n->weight_type != n->type && n->weight_type != FOBQ_F32) return set_err(ctx, FOBQ_EINVAL, "weight_type must be type or F32 (got %d)", n->weight_type);
    if (!finite(n->eps) || n->eps < 0.f) return set_err(ctx, FOBQ_EINVAL, "eps must be finite and >= 0");
    if (n->x_ld < m.cols || (n->residual && n->residual_ld < m.cols) || (n->sum && n->sum_ld < m.cols) || (n->norm && n->norm_ld < m.cols))
        return set_err(ctx, FOBQ_EINVAL, "a row stride is less than cols");
    if (m.rows > 0) {
        const int size = float_size(n->type);
        if (!n->X || !aligned(n->X, size) || !aligned(n->residual, size) || !aligned(n->sum, size) || !aligned(n->norm, size) ||
            !aligned(n->weight, float_size(n->weight_type)))
            return set_err(ctx, FOBQ_EINVAL, "X is NULL, or a matrix is not aligned to its elements");
    }
    *v = NormView{n->X, n->residual, n->weight, n->sum, n->norm, n->x_ld, n->residual_ld, n->sum_ld, n->norm_ld, n->eps, m};
    return FOBQ_OK;
}

static int check_router(fobq_ctx* ctx, const fobq_router* r, const fobq_routing* out, RouteView* v)
{
    if (!r || !out) return set_err(ctx, FOBQ_EINVAL, "router or out is NULL");
    if (r->reserved != 0) return set_err(ctx, FOBQ_EINVAL, "reserved must be 0");
    if (!is_float(r->type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", r->type);
    if (r->score != FOBQ_SOFTMAX && r->score != FOBQ_SIGMOID) return set_err(ctx, FOBQ_EINVAL, "unknown score %d", r->score);
    if (r->experts < 1 || r->experts > MAX_EXPERTS) return set_err(ctx, FOBQ_EINVAL, "experts must be in 1..%d (got %d)", MAX_EXPERTS, r->experts);
    if (r->groups < 1 || r->groups > MAX_GROUPS || r->experts % r->groups != 0)
        return set_err(ctx, FOBQ_EINVAL, "groups must be in 1..%d and divide the experts (got %d)", MAX_GROUPS, r->groups);
    if (r->top_groups < 1 || r->top_groups > r->groups) return set_err(ctx, FOBQ_EINVAL, "top_groups must be in 1..groups (got %d)", r->top_groups);
    if (r->group_top != 1 && r->group_top != 2) return set_err(ctx, FOBQ_EINVAL, "group_top must be 1 or 2 (got %d)", r->group_top);
    if (r->top_k < 1 || r->top_k > MAX_TOP || r->top_k > r->experts / r->groups * r->top_groups)
        return set_err(ctx, FOBQ_EINVAL, "top_k must be in 1..%d and no more than the experts of top_groups groups (got %d)", MAX_TOP, r->top_k);
    if (!finite(r->scale)) return set_err(ctx, FOBQ_EINVAL, "scale must be finite");
    if (r->tokens < 0 || r->tokens > MAX_ROWS || r->tokens * r->top_k >= MAX_SIDE)
        return set_err(ctx, FOBQ_EINVAL, "tokens must be in 0..%lld, and tokens * top_k below %lld (got %lld)", (long long)MAX_ROWS, (long long)MAX_SIDE, (long long)r->tokens);
    if (r->ld < r->experts) return set_err(ctx, FOBQ_EINVAL, "ld (%lld) is less than experts", (long long)r->ld);
    if (!aligned(r->bias, 4)) return set_err(ctx, FOBQ_EINVAL, "bias is not aligned to its elements");
    if (!out->starts || !aligned(out->starts, 4)) return set_err(ctx, FOBQ_EINVAL, "starts is NULL or not aligned to its elements");
    if (r->tokens > 0) {
        if (!r->logits || !aligned(r->logits, float_size(r->type))) return set_err(ctx, FOBQ_EINVAL, "logits is NULL or not aligned to its elements");
        if (!out->chosen || !out->weights || !out->pairs || !out->places || !aligned(out->chosen, 4) || !aligned(out->weights, 4) || !aligned(out->pairs, 4) ||
            !aligned(out->places, 4))
            return set_err(ctx, FOBQ_EINVAL, "a part of the routing is NULL or not aligned to its elements");
    }
    *v = RouteView{r->logits, r->bias, r->ld, (int)r->tokens, r->experts, r->top_k, r->score, r->groups, r->top_groups, r->group_top, r->renormalize, r->scale,
                   out->chosen, out->weights, out->starts, out->pairs, out->places};
    return FOBQ_OK;
}

static int check_experts(fobq_ctx* ctx, const fobq_fp8_matrix* A, const fobq_fp8_experts* B, const int32_t* starts, const int32_t* pairs, int32_t top_k, int64_t rows,
                         int32_t type, int64_t ld, ExpertView* v, ExpertPlan* p)
{
    Fp8View a, b;
    int rc = check_matrix(ctx, A, "A", &a);
    if (rc) return rc;
    if (!B) return set_err(ctx, FOBQ_EINVAL, "B is NULL");
    if (B->reserved != 0) return set_err(ctx, FOBQ_EINVAL, "reserved must be 0");
    if (B->experts < 1 || B->experts > MAX_EXPERTS) return set_err(ctx, FOBQ_EINVAL, "experts must be in 1..%d (got %d)", MAX_EXPERTS, B->experts);
    const fobq_fp8_matrix one{B->values, B->scales, B->rows, B->cols, B->ld, B->ld_scales, B->rows_per_scale, B->format};
    if ((rc = check_matrix(ctx, &one, "B", &b))) return rc;
    if (B->expert_values % 16 != 0 || B->expert_values < 0 || B->expert_scales < 0)
        return set_err(ctx, FOBQ_EINVAL, "expert_values must be a multiple of 16, and neither it nor expert_scales below 0");
    if (a.per != 1) return set_err(ctx, FOBQ_EINVAL, "A must have a scale per row");
    if (a.cols != b.cols) return set_err(ctx, FOBQ_EINVAL, "A has %d columns, B %d", a.cols, b.cols);
    if (a.ld >= MAX_APART || b.ld >= MAX_APART) return set_err(ctx, FOBQ_EINVAL, "rows must be less than %lld bytes apart", (long long)MAX_APART);
    if (rows < 0 || rows > MAX_ROWS) return set_err(ctx, FOBQ_EINVAL, "rows must be in 0..%lld (got %lld)", (long long)MAX_ROWS, (long long)rows);
    if (top_k < 1 || top_k > MAX_TOP) return set_err(ctx, FOBQ_EINVAL, "top_k must be in 1..%d (got %d)", MAX_TOP, top_k);
    if (!pairs && a.rows < rows) return set_err(ctx, FOBQ_EINVAL, "A has %d rows, less than %lld", a.rows, (long long)rows);
    if (!is_float(type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", type);
    if (ld < b.rows) return set_err(ctx, FOBQ_EINVAL, "ld (%lld) is less than the rows of B", (long long)ld);
    *p = expert_plan(ctx ? ctx->cus : 256, rows, B->experts, b.rows, a.cols, type, b.per);
    if (p->tiles * (p->tm == 16 || p->tn == 256 || p->parts == 2 ? 2 : 1) > MAX_TILES)      // (those have 512 threads)
        return set_err(ctx, FOBQ_EINVAL, "Y may have more than %lld tiles of %d", (long long)MAX_TILES, p->tm);
    *v = ExpertView{a, b, B->experts, B->expert_values, B->expert_scales, starts, pairs, top_k, (int)rows, nullptr, type, ld};
    return FOBQ_OK;
}

static int check_sum(fobq_ctx* ctx, int32_t type, int64_t rows, int64_t cols, int64_t ld, int64_t tokens, int32_t top_k, const void* base, int64_t base_ld, int64_t out_ld)
{
    if (!is_float(type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", type);
    if (rows < 0 || rows > MAX_ROWS || tokens < 0 || tokens > MAX_ROWS || cols < 0 || cols >= MAX_SIDE)
        return set_err(ctx, FOBQ_EINVAL, "rows and tokens must be in 0..%lld, cols below %lld", (long long)MAX_ROWS, (long long)MAX_SIDE);
    if (tokens * std::max<int64_t>(1, (cols + 511) / 512) > MAX_ROWS) return set_err(ctx, FOBQ_EINVAL, "tokens times 512 columns must be no more than %lld", (long long)MAX_ROWS);
    if (top_k < 1 || top_k > MAX_TOP) return set_err(ctx, FOBQ_EINVAL, "top_k must be in 1..%d (got %d)", MAX_TOP, top_k);
    if (ld < cols || out_ld < cols || (base && base_ld < cols)) return set_err(ctx, FOBQ_EINVAL, "a row stride is less than cols");
    return FOBQ_OK;
}

int experts_debug_plan(int32_t what, const int64_t* in, int32_t n_in, int64_t* out, int32_t n_out)
{
    auto address = [](int64_t x) { return reinterpret_cast<void*>(static_cast<uintptr_t>(x)); };
    auto whole = [&](int i) { return static_cast<int32_t*>(address(in[i])); };
    if (what == FOBQ_PLAN_ROUTE && n_in == 2 && n_out == 3) {
        if (in[0] < 0 || in[0] > MAX_ROWS || in[1] < 1 || in[1] > MAX_EXPERTS) return FOBQ_EINVAL;
        const RoutePlan p = route_plan(in[0]);
        out[0] = p.parts; out[1] = p.per_part; out[2] = route_workspace(p, (int)in[1]);
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_EXPERTS && n_in == 7 && (n_out == 3 || n_out == 4)) {
        for (int i = 0; i < 5; ++i)
            if (in[i] < (i ? 0 : 16) || in[i] > (i ? i == 2 ? MAX_EXPERTS : MAX_ROWS : 4096)) return FOBQ_EINVAL;
        if (in[2] < 1 || !is_float((int)in[5]) || (in[6] != 1 && in[6] != 128)) return FOBQ_EINVAL;
        const ExpertPlan p = expert_plan((int)in[0], in[1], (int)in[2], in[3], in[4], (int)in[5], (int)in[6]);
        out[0] = p.tm; out[1] = p.tn; out[2] = p.tiles;
        if (n_out == 4) out[3] = p.parts;
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_NORM_CHECK && n_in == 14 && n_out == 1) {
        const fobq_norm n{address(in[9]), address(in[10]), address(in[11]), address(in[12]), address(in[13]), in[2], in[3], in[4], in[5], (int32_t)in[6], (int32_t)in[7],
                          in[8] < 0 ? -1e-6f : in[8] > 0 ? __builtin_inff() : 1e-6f, 0};
        const fobq_fp8_matrix m{address(1 << 20), static_cast<float*>(address(1 << 20)), in[0], in[1], (in[1] + 15) / 16 * 16, in[0], 1, FOBQ_E4M3};
        NormView v;
        out[0] = check_norm(nullptr, &n, &m, &v);
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_ROUTE_CHECK && n_in == 17 && n_out == 1) {
        const fobq_router r{address(in[10]), static_cast<float*>(address(in[11])), in[0], in[1], (int32_t)in[2], (int32_t)in[3], (int32_t)in[4], (int32_t)in[5],
                            (int32_t)in[6], (int32_t)in[7], (int32_t)in[8], 1, 1.f, (int32_t)in[9]};
        const fobq_routing to{whole(12), static_cast<float*>(address(in[13])), whole(14), whole(15), whole(16)};
        RouteView v;
        out[0] = check_router(nullptr, &r, &to, &v);
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_EXPERTS_CHECK && n_in == 15 && n_out == 1) {
        const fobq_fp8_matrix a{address(1 << 20), static_cast<float*>(address(1 << 20)), in[0], in[1], (in[1] + 15) / 16 * 16, in[0], 1, FOBQ_E4M3};
        const fobq_fp8_experts b{address(in[9]), static_cast<float*>(address(in[9])), in[2], in[3], in[4], in[2], in[5], in[6], (int32_t)in[7], (int32_t)in[8], FOBQ_E4M3, 0};
        ExpertView v;
        ExpertPlan p;
        out[0] = check_experts(nullptr, &a, &b, nullptr, whole(10), (int32_t)in[11], in[12], (int32_t)in[13], in[14], &v, &p);
        return FOBQ_OK;
    }
    if (what == FOBQ_PLAN_SUM_CHECK && n_in == 9 && n_out == 1) {
        out[0] = check_sum(nullptr, (int32_t)in[0], in[1], in[2], in[3], in[4], (int32_t)in[5], address(in[6]), in[7], in[8]);
        return FOBQ_OK;
    }
    return FOBQ_EINVAL;
}

}  // namespace fobq

using namespace fobq;

extern "C" {

int fobq_fp8_rms_norm(fobq_ctx* ctx, const fobq_norm* norm, const fobq_fp8_matrix* out)
{
    if (!ctx) return FOBQ_EINVAL;
    NormView v;
    int rc = check_norm(ctx, norm, out, &v);
    if (rc || v.out.rows == 0) return rc;
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_rms_norm(ctx->stream, v, norm->type, norm->weight_type), "norm into 8-bit blocks");
    return FOBQ_OK;
}

int fobq_fp8_swiglu(fobq_ctx* ctx, const void* X, int32_t type, int64_t ld, const fobq_fp8_matrix* out)
{
    if (!ctx) return FOBQ_EINVAL;
    Fp8View v;
    int rc = check_matrix(ctx, out, "out", &v);
    if (rc) return rc;
    if (!is_float(type)) return set_err(ctx, FOBQ_EINVAL, "unknown type %d", type);
    if (v.per != 1) return set_err(ctx, FOBQ_EINVAL, "out must have a scale per row");
    if (ld < 2 * (int64_t)v.cols) return set_err(ctx, FOBQ_EINVAL, "ld (%lld) is less than twice the columns", (long long)ld);
    if (v.rows == 0 || v.cols == 0) return FOBQ_OK;
    if (!X || !aligned(X, float_size(type))) return set_err(ctx, FOBQ_EINVAL, "X is NULL or not aligned to its elements");
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_swiglu(ctx->stream, X, type, ld, v), "gated activation into 8-bit blocks");
    return FOBQ_OK;
}

int fobq_route_workspace(fobq_ctx* ctx, int64_t tokens, int32_t experts, int64_t* bytes)
{
    if (!ctx) return FOBQ_EINVAL;
    if (!bytes || tokens < 0 || tokens > MAX_ROWS || experts < 1 || experts > MAX_EXPERTS)
        return set_err(ctx, FOBQ_EINVAL, "bytes is NULL, tokens not in 0..%lld or experts not in 1..%d", (long long)MAX_ROWS, MAX_EXPERTS);
    *bytes = route_workspace(route_plan(tokens), experts);
    return FOBQ_OK;
}

int fobq_route(fobq_ctx* ctx, const fobq_router* router, const fobq_routing* out, void* work, int64_t work_bytes)
{
    if (!ctx) return FOBQ_EINVAL;
    RouteView v;
    int rc = check_router(ctx, router, out, &v);
    if (rc) return rc;
    const RoutePlan p = route_plan(v.tokens);
    const int64_t need = route_workspace(p, v.experts);
    if (work_bytes < need || (need > 0 && (!work || !aligned(work, 16))))
        return set_err(ctx, FOBQ_EINVAL, "work must be %lld bytes, 16-byte aligned (got %lld)", (long long)need, (long long)work_bytes);
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_route(ctx->stream, p, v, router->type, need ? static_cast<int32_t*>(work) : nullptr), "routing to experts");
    return FOBQ_OK;
}

int fobq_fp8_expert_matmul(fobq_ctx* ctx, const fobq_fp8_matrix* A, const fobq_fp8_experts* B, const int32_t* starts, const int32_t* pairs, int32_t top_k,
                           int64_t rows, void* Y, int32_t type, int64_t ld)
{
    if (!ctx) return FOBQ_EINVAL;
    ExpertView v;
    ExpertPlan p;
    int rc = check_experts(ctx, A, B, starts, pairs, top_k, rows, type, ld, &v, &p);
    if (rc) return rc;
    if (v.rows == 0 || v.a.rows == 0 || v.b.rows == 0) return FOBQ_OK;
    if (!starts || !aligned(starts, 4) || !aligned(pairs, 4)) return set_err(ctx, FOBQ_EINVAL, "starts is NULL, or starts or pairs not aligned to its elements");
    if (!Y || !aligned(Y, float_size(type))) return set_err(ctx, FOBQ_EINVAL, "Y is NULL or not aligned to its elements");
    v.y = Y;
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    FOBQ_TRY(launch_expert_matmul(ctx->stream, p, v), "products of the experts' rows");
    return FOBQ_OK;
}

int fobq_expert_sum(fobq_ctx* ctx, const void* Y, int32_t type, int64_t rows, int64_t cols, int64_t ld, const float* weights, const int32_t* places,
                    int64_t tokens, int32_t top_k, const void* base, int64_t base_ld, void* out, int64_t out_ld)
{
    if (!ctx) return FOBQ_EINVAL;
    int rc = check_sum(ctx, type, rows, cols, ld, tokens, top_k, base, base_ld, out_ld);
    if (rc) return rc;
    if (tokens == 0 || cols == 0) return FOBQ_OK;
    const int size = float_size(type);
    if ((rows > 0 && !Y) || !out || !weights || !places || !aligned(Y, size) || !aligned(out, size) || !aligned(base, size) || !aligned(weights, 4) || !aligned(places, 4))
        return set_err(ctx, FOBQ_EINVAL, "Y, out, weights or places is NULL, or something is not aligned to its elements");
    DeviceGuard g(ctx->device);
    if ((rc = enter(ctx, g))) return rc;
    const ExpertSum v{Y, ld, (int)rows, weights, places, (int)tokens, top_k, cols, base, base_ld, out, out_ld};
    FOBQ_TRY(launch_expert_sum(ctx->stream, v, type), "sum of the experts' rows");
    return FOBQ_OK;
}

}  // extern "C"
