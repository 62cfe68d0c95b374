// Routing of tokens to experts, and the weighted sum of the experts' rows behind it.
//
// A wavefront has a token: its scores, the choice of groups and of experts, and the weights never leave registers.  A lane has neighbouring
// experts, so that the lowest lane among equal ones has the lowest expert; with groups, 64 / groups lanes (rounded down to a power of two) have a group.  The
// largest key is found top_k times, by the bits of the keys, which order as the keys do.
//
// Where the rows lie is a counting sort that keeps the pairs' order.  A token has an expert once at most, so that the experts' rows among 64
// tokens are bits of a word, set in any order, and a pair's rank is the number of bits below its token's: no result depends on the order
// in which workgroups or atomics run.
#include "lowbit.h"

#include <algorithm>
#include <type_traits>

namespace fobq {

constexpr int ROUTE_WAVES = 16;

template <class F>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, F f)
{
    auto dpp = [](uint32_t v, auto ctrl) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, decltype(ctrl)::value, 0xf, 0xf, true); };
    x = f(x, dpp(x, std::integral_constant<int, 0xB1>()));
    x = f(x, dpp(x, std::integral_constant<int, 0x4E>()));
    x = f(x, dpp(x, std::integral_constant<int, 0x141>()));
    x = f(x, dpp(x, std::integral_constant<int, 0x140>()));
    auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return f(r[0], r[1]);
}
__device__ __forceinline__ uint32_t wave_most(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)over_wave(x, [](uint32_t a, uint32_t b) { return max(a, b); }));
}
__device__ __forceinline__ float wave_sum(float x)
{
    return __uint_as_float(over_wave(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// Bits that order as the values do, above 0 for all but -Inf, which is 0 as what is not there.  (-0 and 0 are alike: + 0 makes both 0.)
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return x == -__builtin_inff() ? 0u : (b >> 31 ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ uint64_t order_of(double x)
{
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
    return x == -__builtin_inf() ? 0ull : (b >> 63 ? ~b : b | 0x8000000000000000ull);
}

// The lane that has the largest, the lowest of several; -1 if all are 0.
__device__ __forceinline__ int lane_of_most(uint32_t x)
{
    const uint32_t most = wave_most(x);
    return most == 0 ? -1 : __builtin_ctzll(__ballot(x == most));
}
__device__ __forceinline__ int lane_of_most(uint64_t x)
{
    const uint32_t hi = (uint32_t)(x >> 32), most = wave_most(hi);
    if (most == 0) return -1;                                // (the bits of a number that is not 0 have a high half)
    unsigned long long have = __ballot(hi == most);
    if (have & (have - 1)) {
        const uint32_t low = wave_most(hi == most ? (uint32_t)x : 0u);
        have = __ballot(hi == most && (uint32_t)x == low);
    }
    return __builtin_ctzll(have);
}

// key[j]: what is chosen by, -Inf where an expert is none; the lane's group has `wide` lanes, its groups are `groups`.  Lane s gets the index, lane * V + j,
// in slot s, or -1.
template <int V, class K>
__device__ __forceinline__ int choose(const K (&key)[V], const RouteView& g, int wide)
{
    using U = decltype(order_of(K()));
    const int lane = threadIdx.x & 63;
    U at[V];
#pragma unroll
    for (int j = 0; j < V; ++j) at[j] = order_of(key[j]);
    if (g.groups > 1) {
        const K none = -(K)__builtin_inf();
        K first = none, second = none;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            second = max(second, min(first, key[j]));
            first = max(first, key[j]);
        }
        for (int off = 1; off < wide; off <<= 1) {
            const K f = __shfl_xor(first, off), s = __shfl_xor(second, off);
            second = max(max(second, s), min(first, f));
            first = max(first, f);
        }
        const U level = order_of(g.group_top == 2 && second != none ? first + second : first);
        const int mine = lane / wide;
        int better = 0;
        for (int o = 0; o < g.groups; ++o) {
            const U other = __shfl(level, o * wide);
            better += other > level || (other == level && o < mine);
        }
        if (better >= g.top_groups)
#pragma unroll
            for (int j = 0; j < V; ++j) at[j] = 0;
    }
    int got = -1;
    for (int s = 0; s < g.top; ++s) {
        U best = at[0];
        int where = 0;
#pragma unroll
        for (int j = 1; j < V; ++j)
            if (at[j] > best) best = at[j], where = j;
        const int from = lane_of_most(best);
        if (from < 0) break;
        const int index = __shfl(lane * V + where, from);
        if (lane == s) got = index;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (lane * V + j == index) at[j] = 0;
    }
    return got;
}

// A token's experts and weights, lane s those of slot s.
struct Choice { int expert; float weight; };
template <class T, int V>
__device__ __forceinline__ Choice route_token(const RouteView& g, int64_t token, int wide)
{
    const int lane = threadIdx.x & 63, each = g.experts / g.groups, mine = lane / wide;
    // the lane's experts are first .. first + there - 1
    const int in_group = (lane - mine * wide) * V, first = mine * each + in_group, there = mine < g.groups ? min(V, each - in_group) : 0;
    const T* x = static_cast<const T*>(g.logits) + token * g.ld + first;
    const float none = -__builtin_inff();
    float logit[V], bias[V];
    bool bad = false;
    float most = none;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        logit[j] = j < there ? (float)x[j] : none;
        bias[j] = j < there && g.bias ? g.bias[first + j] : 0.f;
        bad |= logit[j] != logit[j] || !(bias[j] <= 3.402823466e38f) || (g.score == FOBQ_SOFTMAX && logit[j] == __builtin_inff());
        most = fmaxf(most, logit[j]);
    }
    if (__ballot(bad)) return Choice{lane, __builtin_nanf("")};
    most = __uint_as_float(over_wave(__float_as_uint(most), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
    int got;
    if (!g.bias && (g.groups == 1 || g.group_top == 1)) {
        got = choose<V>(logit, g, wide);
    } else {
        double key[V], total = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const double v = logit[j];
            key[j] = logit[j] == none ? 0.0 : g.score == FOBQ_SOFTMAX ? exp(v - (double)most) : 1.0 / (1.0 + exp(-v));
            total += key[j];
        }
        if (g.score == FOBQ_SOFTMAX) {
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off);
        } else {
            total = 1.0;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = logit[j] == none ? -__builtin_inf() : key[j] / total + (double)bias[j];      // (a bias of -Inf: never)
        got = choose<V>(key, g, wide);
    }
    // the slot's logit, from the lane that has it
    const int from = got < 0 ? 0 : got / V;
    float z = none;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float v = __shfl(logit[j], from);
        if (got >= 0 && got - from * V == j) z = v;
    }
    const int owner = from / wide, expert = got < 0 ? -1 : owner * each + (got - owner * wide * V);
    float p = 0.f;
    if (g.renormalize) {
        // relative to the largest: also where the scores themselves are too small for fp32
        const float top = __uint_as_float(over_wave(__float_as_uint(z), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
        if (got >= 0) {
            if (g.score == FOBQ_SOFTMAX) p = expf(z - top);
            else if (top > 0.f) p = (1.f + expf(-top)) / (1.f + expf(-z));
            else p = expf(z - top) * ((1.f + expf(top)) / (1.f + expf(z)));
        }
        p /= wave_sum(p);
    } else if (g.score == FOBQ_SOFTMAX) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) sum += logit[j] == none ? 0.f : expf(logit[j] - most);
        sum = wave_sum(sum);
        if (got >= 0) p = expf(z - most) / sum;
    } else if (got >= 0) {
        p = 1.f / (1.f + expf(-z));
    }
    return Choice{expert, got < 0 ? 0.f : g.scale * p};
}

// Tokens [t0, t1) of a workgroup.  LDS: base, the packed row of each expert's next one; seen, the tokens of 64 that have it.
struct RouteShared { int count[1024]; int base[1025]; uint32_t seen[1024][2]; int sums[ROUTE_WAVES]; };

template <class T, int V>
__device__ __forceinline__ void route_tokens(RouteShared& sh, const RouteView& g, int64_t t0, int64_t t1)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int e = threadIdx.x; e < g.experts; e += 64 * ROUTE_WAVES) sh.count[e] = 0;
    __syncthreads();
    int wide = 64;
    while (wide * g.groups > 64) wide >>= 1;
    for (int64_t t = t0 + wave; t < t1; t += ROUTE_WAVES) {
        const Choice c = route_token<T, V>(g, t, wide);
        if (lane < g.top) {
            g.chosen[t * g.top + lane] = c.expert;
            g.weights[t * g.top + lane] = c.weight;
            if (c.expert >= 0) atomicAdd(&sh.count[c.expert], 1);
        }
    }
    __syncthreads();
}

// From the number of each expert's rows (of all tokens, and of those in front of t0) where they lie; then those of tokens [t0, t1).  Every workgroup
// has the same starts; workgroup `part` of `parts` writes some of what is -1.
__device__ __forceinline__ void route_places(RouteShared& sh, const RouteView& g, int64_t t0, int64_t t1, int mine, int before, int part, int parts)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // thread e has expert e: an ascending sum over the threads
    int sum = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(sum, off);
        if (lane >= off) sum += v;
    }
    if (lane == 63) sh.sums[wave] = sum;
    __syncthreads();
    int at = sum - mine;
    for (int w = 0; w < wave; ++w) at += sh.sums[w];
    if (tid < g.experts) {
        sh.base[tid] = at + before;
        sh.seen[tid][0] = sh.seen[tid][1] = 0;
        if (part == 0) g.starts[tid] = at;
        if (tid == g.experts - 1) {
            sh.base[1024] = at + mine;
            if (part == 0) g.starts[g.experts] = at + mine;
        }
    }
    __syncthreads();
    const int64_t pairs = (int64_t)g.tokens * g.top;
    for (int64_t i = sh.base[1024] + (int64_t)part * (64 * ROUTE_WAVES) + tid; i < pairs; i += (int64_t)parts * (64 * ROUTE_WAVES)) g.pairs[i] = -1;
    for (int64_t t = t0; t < t1; t += 64) {
        const int n = (int)min((int64_t)64, t1 - t) * g.top;
        for (int i = tid; i < n; i += 64 * ROUTE_WAVES) {
            const int e = g.chosen[t * g.top + i], bit = i / g.top;
            if (e >= 0) atomicOr(&sh.seen[e][bit >> 5], 1u << (bit & 31));
        }
        __syncthreads();
        for (int i = tid; i < n; i += 64 * ROUTE_WAVES) {
            const int e = g.chosen[t * g.top + i], bit = i / g.top;
            int place = -1;
            if (e >= 0) {
                const uint32_t below = (1u << (bit & 31)) - 1;
                place = sh.base[e] + (bit < 32 ? __popc(sh.seen[e][0] & below) : __popc(sh.seen[e][0]) + __popc(sh.seen[e][1] & below));
                g.pairs[place] = (int)(t * g.top + i);
            }
            g.places[t * g.top + i] = place;
        }
        __syncthreads();
        if (tid < g.experts) {
            sh.base[tid] += __popc(sh.seen[tid][0]) + __popc(sh.seen[tid][1]);
            sh.seen[tid][0] = sh.seen[tid][1] = 0;
        }
        __syncthreads();
    }
}

// All of it where one workgroup has the tokens; otherwise the choice, and how often each expert is in it.
template <class T, int V>
__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_choose_kernel(RouteView g, RoutePlan p, int32_t* __restrict__ work)
{
    __shared__ RouteShared sh;
    const int64_t t0 = (int64_t)blockIdx.x * p.per_part, t1 = min((int64_t)g.tokens, t0 + p.per_part);
    route_tokens<T, V>(sh, g, t0, t1);
    const int tid = threadIdx.x;
    if (p.parts == 1) {
        // (the workgroup's own stores of `chosen` are seen behind its barrier)
        route_places(sh, g, t0, t1, tid < g.experts ? sh.count[tid] : 0, 0, 0, 1);
    } else if (tid < g.experts) {
        work[(int64_t)blockIdx.x * g.experts + tid] = sh.count[tid];
    }
}

__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_places_kernel(RouteView g, RoutePlan p, const int32_t* __restrict__ work)
{
    __shared__ RouteShared sh;
    const int tid = threadIdx.x, part = blockIdx.x;
    const int64_t t0 = (int64_t)part * p.per_part, t1 = min((int64_t)g.tokens, t0 + p.per_part);
    int all = 0, before = 0;
    if (tid < g.experts)
        for (int w = 0; w < p.parts; ++w) {
            const int n = work[(int64_t)w * g.experts + tid];
            all += n;
            before += w < part ? n : 0;
        }
    route_places(sh, g, t0, t1, all, before, part, p.parts);
}

// A wavefront has 512 columns of a token: where its rows lie, and their weights, are the same for all lanes.
template <class T>
__global__ __launch_bounds__(256) void expert_sum_kernel(ExpertSum g, unsigned across)
{
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), token = item / across;
    if (token >= g.tokens) return;
    const int64_t col = (item - token * across) * 512 + 8 * lane;
    const int left = (int)min((int64_t)8, g.cols - col);
    if (left <= 0) return;
    const T* y = static_cast<const T*>(g.y) + col;
    auto load = [&](const T* p, float* x) {
        if (left == 8) load8(p, x);
        else
            for (int i = 0; i < 8; ++i) x[i] = i < left ? (float)p[i] : 0.f;
    };
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (g.base) load(static_cast<const T*>(g.base) + token * g.base_ld + col, sum);
    for (int s = 0; s < g.top; ++s) {
        const int place = g.places[token * g.top + s];
        if ((unsigned)place >= (unsigned)g.rows) continue;
        const float w = g.weights[token * g.top + s];
        float x[8];
        load(y + (int64_t)place * g.ld, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, x[i], sum[i]);
    }
    T* out = static_cast<T*>(g.out) + token * g.out_ld + col;
    if (left == 8) store8(out, sum);
    else
        for (int i = 0; i < left; ++i) out[i] = (T)sum[i];
}

RoutePlan route_plan(int64_t tokens)
{
    const int64_t per = std::max<int64_t>(1, (tokens + 64 * 256 - 1) / (64 * 256)) * 64;
    return RoutePlan{(int)std::max<int64_t>(1, (tokens + per - 1) / per), (int)per};
}

int64_t route_workspace(const RoutePlan& p, int experts) { return p.parts > 1 ? (int64_t)p.parts * experts * (int64_t)sizeof(int32_t) : 0; }

template <class T>
static hipError_t route_of(hipStream_t s, const RoutePlan& p, const RouteView& g, int32_t* work)
{
    int wide = 64;
    while (wide * g.groups > 64) wide >>= 1;
    const int each = (g.experts / g.groups + wide - 1) / wide;         // experts of a lane
    const dim3 grid((unsigned)p.parts), block(64 * ROUTE_WAVES);
    if (each <= 1) hipLaunchKernelGGL((route_choose_kernel<T, 1>), grid, block, 0, s, g, p, work);
    else if (each <= 2) hipLaunchKernelGGL((route_choose_kernel<T, 2>), grid, block, 0, s, g, p, work);
    else if (each <= 4) hipLaunchKernelGGL((route_choose_kernel<T, 4>), grid, block, 0, s, g, p, work);
    else if (each <= 8) hipLaunchKernelGGL((route_choose_kernel<T, 8>), grid, block, 0, s, g, p, work);
    else if (each <= 16) hipLaunchKernelGGL((route_choose_kernel<T, 16>), grid, block, 0, s, g, p, work);
    else hipLaunchKernelGGL((route_choose_kernel<T, 32>), grid, block, 0, s, g, p, work);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL(route_places_kernel, grid, block, 0, s, g, p, work);
    return hipGetLastError();
}

hipError_t launch_route(hipStream_t s, const RoutePlan& p, const RouteView& g, int type, int32_t* work)
{
    if (type == FOBQ_F32) return route_of<float>(s, p, g, work);
    return type == FOBQ_BF16 ? route_of<bf16_t>(s, p, g, work) : route_of<f16_t>(s, p, g, work);
}

template <class T>
static hipError_t sum_of(hipStream_t s, const ExpertSum& g)
{
    const unsigned across = (unsigned)((g.cols + 511) / 512);
    hipLaunchKernelGGL((expert_sum_kernel<T>), dim3((unsigned)(((int64_t)g.tokens * across + 3) / 4)), dim3(256), 0, s, g, across);
    return hipGetLastError();
}

hipError_t launch_expert_sum(hipStream_t s, const ExpertSum& g, int type)
{
    if (type == FOBQ_F32) return sum_of<float>(s, g);
    return type == FOBQ_BF16 ? sum_of<bf16_t>(s, g) : sum_of<f16_t>(s, g);
}

}  // namespace fobq
