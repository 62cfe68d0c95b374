// Routing of tokens to experts, and the weighted sum of the experts' rows behind it.
//
// Up to 256 experts in groups that lanes can share: four tokens a wavefront, sixteen lanes a token, a key and its expert in one word
// of 31 bits (route_tokens_by_four).  Otherwise a wavefront has a token, a lane neighbouring experts, so that the lowest lane among equal ones has the lowest expert; with groups,
// 64 / groups lanes (rounded down to a power of two) have a group.  Scores, the choice and the weights never leave registers; the largest key is found top_k times, by bits that
// order as the keys do.
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
__device__ __forceinline__ int lane_of_most(uint32_t x, uint32_t& most)
{
    most = wave_most(x);
    return most == 0 ? -1 : __builtin_ctzll(__ballot(x == most));
}
__device__ __forceinline__ int lane_of_most(uint64_t x, uint64_t& most)
{
    const uint32_t hi = (uint32_t)(x >> 32), top = wave_most(hi);
    if (top == 0) return -1;                                 // (the bits of a number that is not 0 have a high half)
    const uint32_t low = wave_most(hi == top ? (uint32_t)x : 0u);
    most = (uint64_t)top << 32 | low;
    return __builtin_ctzll(__ballot(x == most));
}

__device__ __forceinline__ float value_of(uint32_t bits) { return __uint_as_float(bits >> 31 ? bits & 0x7fffffffu : ~bits); }

// f over the `wide` lanes of a group, a power of two up to 32, the result in all of them.  (Lanes at mirrored places stand for those at a distance: what they hold
// is the same over each half by then.)
template <class F>
__device__ __forceinline__ void over_group(int wide, F f)
{
    auto dpp = [](auto ctrl) { return [](float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); }; };
    if (wide > 1) f(dpp(std::integral_constant<int, 0xB1>()));
    if (wide > 2) f(dpp(std::integral_constant<int, 0x4E>()));
    if (wide > 4) f(dpp(std::integral_constant<int, 0x141>()));
    if (wide > 8) f(dpp(std::integral_constant<int, 0x140>()));
    if (wide > 16) f([](float v) { return __shfl_xor(v, 16); });
}
template <class F>
__device__ __forceinline__ void over_group(int wide, F f, double)
{
    for (int off = 1; off < wide; off <<= 1) f([off](double v) { return __shfl_xor(v, off); });
}

// What a group's two largest keys count as.  In fp32 it stays finite: -Inf is a group without experts, and biases near the ends of fp32 would make others that too.
__device__ __forceinline__ float level_of(float first, float second) { return __builtin_amdgcn_fmed3f(first + second, -3.402823466e38f, 3.402823466e38f); }
__device__ __forceinline__ double level_of(double first, double second) { return first + second; }

// What is the same for all tokens of a wavefront: a lane's experts are first .. first + there - 1, group `mine` of `wide` lanes has `each`.
template <int V> struct RouteLane { int first, there, mine, wide, each; float bias[V], most_bias; bool bad; };

// key[j]: what is chosen by, -Inf where an expert is none.  Lane s gets the index, lane * V + j, in slot s, or -1.  With slack > 0 keys and groups that are that
// near each other may be in either order: `sure` then says that there were none, but for equal ones of the same logit and bias; and that nothing else is that near
// the last one chosen, looked at or not (behind equals there may be a larger key that these do not show).
template <int V, class K>
__device__ __forceinline__ int choose(const K (&key)[V], const RouteView& g, const RouteLane<V>& l, float slack, const float (&logit)[V], bool& sure)
{
    using U = decltype(order_of(K()));
    constexpr bool SORTED = V <= 4 && sizeof(K) == 4;        // a lane's keys in descending order: the largest is the first
    const int lane = threadIdx.x & 63;
    U at[V];
    int who[V];
#pragma unroll
    for (int j = 0; j < V; ++j) at[j] = order_of(key[j]), who[j] = lane * V + j;
    bool kept = true;
    if (g.groups > 1) {
        const K none = -(K)__builtin_inf();
        K first = none, second = none;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            second = max(second, min(first, key[j]));
            first = max(first, key[j]);
        }
        auto join = [&](auto other) {
            const K f = other(first), s = other(second);
            second = max(max(second, s), min(first, f));
            first = max(first, f);
        };
        if constexpr (sizeof(K) == 4) over_group(l.wide, join);
        else over_group(l.wide, join, 0.0);
        const U level = order_of(g.group_top == 2 && second != none ? level_of(first, second) : first);
        int better = 0;
        for (int o = 0; o < g.groups; ++o) {
            U other;
            if constexpr (sizeof(K) == 4) other = (U)__builtin_amdgcn_readlane((int)level, o * l.wide);
            else other = __shfl(level, o * l.wide);
            better += other > level || (other == level && o < l.mine);
        }
        kept = better < g.top_groups;
        if (!kept)
#pragma unroll
            for (int j = 0; j < V; ++j) at[j] = 0;
        if constexpr (sizeof(K) == 4) {
            if (slack > 0.f && g.top_groups < g.groups) {
                // the last group that is kept, and the first that is not
                const bool real = l.mine < g.groups;
                const int in = __builtin_ctzll(__ballot(real && better == g.top_groups - 1)), out = __builtin_ctzll(__ballot(real && better == g.top_groups));
                const uint32_t kept = (uint32_t)__builtin_amdgcn_readlane((int)level, in), left = (uint32_t)__builtin_amdgcn_readlane((int)level, out);
                if (left != 0 && value_of(kept) - value_of(left) <= 3.f * slack) sure = false;
            }
        }
    }
    if constexpr (SORTED) {
        // (neighbours in turn, only where the later one is larger: equal ones stay in their order)
#pragma unroll
        for (int round = 0; round < V; ++round)
#pragma unroll
            for (int j = round & 1; j + 1 < V; j += 2) {
                const bool swap = at[j + 1] > at[j];
                const U a = at[j], b = at[j + 1];
                const int wa = who[j], wb = who[j + 1];
                at[j] = swap ? b : a, at[j + 1] = swap ? a : b;
                who[j] = swap ? wb : wa, who[j + 1] = swap ? wa : wb;
            }
    }
    int got = -1, before = 0;
    U last = 0;
    const int looks = slack > 0.f ? g.top + 1 : g.top;       // (one more: whether the last one is sure)
    for (int s = 0; s < looks; ++s) {
        U best = at[0];
        int where = who[0];
        if constexpr (!SORTED) {
#pragma unroll
            for (int j = 1; j < V; ++j)
                if (at[j] > best) best = at[j], where = who[j];
        }
        U most = 0;
        const int from = lane_of_most(best, most);
        if (from < 0) break;
        const int index = __builtin_amdgcn_readlane(where, from);
        if constexpr (sizeof(K) == 4) {
            if (slack > 0.f && s > 0 && value_of(last) - value_of(most) <= slack) {
                auto of = [&](int i, const float (&v)[V]) {
                    float x = 0.f;
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (i % V == j) x = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[j]), i / V));
                    return x;
                };
                const float z = of(before, logit), b = of(before, l.bias);
                if (s < g.top) {
                    if (!(of(index, logit) == z && of(index, l.bias) == b)) sure = false;
                } else {
                    const float v = value_of(last);
                    bool other = false;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        // (sorted ones are not at their experts' places any more; those chosen earlier have been compared, which does no harm again)
                        const bool close = SORTED ? kept && fabsf((float)key[j] - v) <= slack : at[j] != 0 && v - value_of((uint32_t)at[j]) <= slack;
                        other |= close && !(logit[j] == z && l.bias[j] == b);
                    }
                    if (__ballot(other)) sure = false;
                }
            }
        }
        if (lane == s && s < g.top) got = index;
        last = most;
        before = index;
        if constexpr (SORTED) {
            if (lane == from) {
#pragma unroll
                for (int j = 0; j + 1 < V; ++j) at[j] = at[j + 1], who[j] = who[j + 1];
                at[V - 1] = 0;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (who[j] == index) at[j] = 0;
        }
    }
    return got;
}

template <int V, int LANES>
__device__ __forceinline__ RouteLane<V> route_lane(const RouteView& g)
{
    const int lane = threadIdx.x & (LANES - 1);
    RouteLane<V> l;
    l.wide = LANES;
    while (l.wide * g.groups > LANES) l.wide >>= 1;
    l.each = g.experts / g.groups;
    l.mine = lane / l.wide;
    const int in_group = (lane - l.mine * l.wide) * V;
    l.first = l.mine * l.each + in_group;
    l.there = l.mine < g.groups ? min(V, max(0, l.each - in_group)) : 0;
    bool bad = false;
    float most = 0.f;
    // (all loads before the first use: a wait for each took 15 us)
#pragma unroll
    for (int j = 0; j < V; ++j) l.bias[j] = 0.f;
    if (g.bias) {
        if (l.there == V) {
            __builtin_memcpy(l.bias, g.bias + l.first, sizeof l.bias);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < l.there) l.bias[j] = g.bias[l.first + j];
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        bad |= !(l.bias[j] <= 3.402823466e38f);
        if (l.bias[j] != -__builtin_inff()) most = fmaxf(most, fabsf(l.bias[j]));
    }
    l.bad = __ballot(bad) != 0;
    l.most_bias = __uint_as_float(wave_most(__float_as_uint(most)));
    return l;
}

// the lane's logits of a token
template <class T, int V>
__device__ __forceinline__ void route_logits(const RouteView& g, const RouteLane<V>& l, int64_t token, T* x)
{
    const T* src = static_cast<const T*>(g.logits) + token * g.ld + l.first;
    if (l.there == V) {
        __builtin_memcpy(x, src, V * sizeof(T));
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = j < l.there ? src[j] : (T)-__builtin_inff();
    }
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(1.44269504f * x); }

// exp(x) to 3 units for x that is not positive (0 from -200 on): 2^t 2^rest, t the product with log2(e) rounded to fp32, rest what that leaves out.
__device__ __forceinline__ float exp_fine(float x)
{
    x = fmaxf(x, -200.f);
    const float t = 1.44269504f * x, rest = fmaf(1.92596299e-8f, x, fmaf(1.44269504f, x, -t)), e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, 0.693147181f * rest, e);
}

// A slot's weight from its logit z (-Inf: none), before the scale.  over(x) and sum(x): the largest and the sum over the token's lanes; most and total: the row's
// largest logit and the sum of exp(x - most), for a softmax that is not renormalized.
template <class Over, class Sum>
__device__ __forceinline__ float route_weight(const RouteView& g, float z, float most, float total, Over over, Sum sum)
{
    const bool there = z != -__builtin_inff();
    float p = 0.f;
    if (g.score == FOBQ_SOFTMAX) {
        const float top = g.renormalize ? over(z) : most;
        if (there) p = exp_fine(z - top);
        return p / (g.renormalize ? sum(p) : total);
    }
    const float e = exp_fine(-fabsf(z));
    if (there) p = (z < 0.f ? e : 1.f) / (1.f + e);
    if (!g.renormalize) return p;
    const float top = over(z);
    if (__ballot(top < -60.f)) {
        // relative to the largest, where the scores themselves are too small for fp32
        if (there && top < -60.f) p = exp_fine(z - top);
    }
    return p / sum(p);
}

// A token's experts and weights, lane s those of slot s.  SCORED: scores are compared, not logits.
struct Choice { int expert; float weight; };
template <class T, int V, bool SCORED>
__device__ __forceinline__ Choice route_token(const RouteView& g, const RouteLane<V>& l, const T* raw)
{
    const int lane = threadIdx.x & 63;
    const float none = -__builtin_inff();
    float logit[V], most = none;
    bool bad = false;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        logit[j] = (float)raw[j];
        bad |= logit[j] != logit[j] || (g.score == FOBQ_SOFTMAX && logit[j] == __builtin_inff());
        most = fmaxf(most, logit[j]);
    }
    if (l.bad || __ballot(bad)) return Choice{lane, __builtin_nanf("")};
    if (g.score == FOBQ_SOFTMAX) most = value_of(wave_most(order_of(most)));          // (no expert at all: NaN, which nothing reads)
    int got;
    bool sure = true;
    if constexpr (!SCORED) {
        got = choose<V>(logit, g, l, 0.f, logit, sure);
    } else {
        // In fp32 first.  A score is off by less than 40 units of the largest one, the sum with a bias by one unit of either more: keys that are
        // apart by more than twice that are in the order that 64 bits have.  Tokens with nearer ones (some in a thousand; nearly all of them beside finite biases far from the
        // others, as masks of -1e9) are looked at in 64 bits.
        float key[V], total = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            key[j] = g.score == FOBQ_SOFTMAX ? exp_of(logit[j] - most) : __builtin_amdgcn_rcpf(1.f + exp_of(-logit[j]));
            if (logit[j] == none) key[j] = 0.f;
            total += key[j];
        }
        const float inv = g.score == FOBQ_SOFTMAX ? __builtin_amdgcn_rcpf(wave_sum(total)) : 1.f;      // (also the largest score, or more)
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = logit[j] == none ? none : fmaf(key[j], inv, l.bias[j]);
        got = choose<V>(key, g, l, 0x1p-24f * (100.f * inv + 4.f * l.most_bias), logit, sure);
        if (!sure) {
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
            for (int j = 0; j < V; ++j) key[j] = logit[j] == none ? -__builtin_inf() : key[j] / total + (double)l.bias[j];     // (a bias of -Inf: never)
            got = choose<V>(key, g, l, 0.f, logit, sure);
        }
    }
    // the slot's logit, from the lane that has it
    const int from = got < 0 ? 0 : got / V;
    float z = none;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float v = __shfl(logit[j], from);
        if (got >= 0 && got - from * V == j) z = v;
    }
    const int owner = from / l.wide, expert = got < 0 ? -1 : owner * l.each + (got - owner * l.wide * V);
    float total = 0.f;
    if (g.score == FOBQ_SOFTMAX && !g.renormalize) {
#pragma unroll
        for (int j = 0; j < V; ++j) total += logit[j] == none ? 0.f : exp_fine(logit[j] - most);
        total = wave_sum(total);
    }
    const float p = route_weight(g, z, most, total, [](float x) { return value_of(wave_most(order_of(x))); }, [](float x) { return wave_sum(x); });
    return Choice{expert, got < 0 ? 0.f : g.scale * p};
}

// LDS of a workgroup.  base: the packed row of each expert's next one; seen: the tokens of 64 that have it; picked: those tokens' experts.
struct RouteShared { int count[1024], before[1024], base[1025]; uint32_t seen[1024][2]; int picked[64 * 32]; int sums[ROUTE_WAVES]; };

// The choice for tokens [t0, t1), and how often each expert is in it.
template <class T, int V, bool SCORED>
__device__ __forceinline__ void route_tokens(RouteShared& sh, const RouteView& g, int64_t t0, int64_t t1)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RouteLane<V> l = route_lane<V, 64>(g);
    sh.count[threadIdx.x] = 0;
    T raw[V], next[V];
    if (t0 + wave < t1) route_logits<T, V>(g, l, t0 + wave, raw);
    __syncthreads();
    for (int64_t t = t0 + wave; t < t1; t += ROUTE_WAVES) {
        if (t + ROUTE_WAVES < t1) route_logits<T, V>(g, l, t + ROUTE_WAVES, next);
        const Choice c = route_token<T, V, SCORED>(g, l, raw);
        if (lane < g.top) {
            g.chosen[t * g.top + lane] = c.expert;
            g.weights[t * g.top + lane] = c.weight;
            sh.picked[(int)(t - t0) % 64 * g.top + lane] = c.expert;
            if (c.expert >= 0) atomicAdd(&sh.count[c.expert], 1);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) raw[j] = next[j];
    }
    __syncthreads();
}

// ---- four tokens a wavefront -----------------------------------------------------------------------------------
// A token has 16 lanes, up to 16 experts each.  What is chosen by becomes a word of 31 bits: the key on a grid of 2^23 steps over the range that keys can
// have (logits: 16 below the largest), and below it the expert's number from behind, so that one maximum says which it is and the next one is the largest of
// what is below it: with all words below 2^31, word - last is at least 2^31 for those alone.  Two instructions a word and choice, where one
// token at a time took twenty.  Tokens whose order that grid, or fp32, does not decide are done again by a wavefront of their own.
template <class F>
__device__ __forceinline__ uint32_t over_row(uint32_t x, F f)
{
    auto dpp = [](uint32_t v, auto ctrl) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, decltype(ctrl)::value, 0xf, 0xf, true); };
    x = f(x, dpp(x, std::integral_constant<int, 0xB1>()));
    x = f(x, dpp(x, std::integral_constant<int, 0x4E>()));
    x = f(x, dpp(x, std::integral_constant<int, 0x141>()));
    return f(x, dpp(x, std::integral_constant<int, 0x140>()));
}
__device__ __forceinline__ uint32_t row_most(uint32_t x) { return over_row(x, [](uint32_t a, uint32_t b) { return max(a, b); }); }
__device__ __forceinline__ uint32_t row_least(uint32_t x) { return over_row(x, [](uint32_t a, uint32_t b) { return min(a, b); }); }
__device__ __forceinline__ float row_most(float x)
{
    return __uint_as_float(over_row(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float row_sum(float x)
{
    return __uint_as_float(over_row(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
constexpr int ROW_TOP = 14;                                  // the choices that 16 lanes can hold, and two more

// A score in 64 bits, times `total` for a softmax.
__device__ __forceinline__ double score64(const RouteView& g, float logit, float most)
{
    const double v = logit;
    return g.score == FOBQ_SOFTMAX ? exp(v - (double)most) : 1.0 / (1.0 + exp(-v));
}

// In 64 bits, for the few tokens that fp32 does not decide: the sum of a softmax's exponentials (1 for a sigmoid), and, if the groups are asked for, whether a lane's
// group is kept.  One expert of a lane at a time, from memory.
template <class T, int V>
__device__ __forceinline__ double route_row64(const RouteView& g, int first, int there, int mine, int wide, int64_t token, float most, bool groups, bool& kept)
{
    const double none = -__builtin_inf();
    double total = 1.0, one = none, two = none;
    if (g.score == FOBQ_SOFTMAX) {
        total = 0.0;
#pragma unroll 1
        for (int j = 0; j < there; ++j) total += score64(g, (float)static_cast<const T*>(g.logits)[token * g.ld + first + j], most);
        for (int off = 1; off < 16; off <<= 1) total += __shfl_xor(total, off);
    }
    if (!groups) return total;
#pragma unroll 1
    for (int j = 0; j < there; ++j) {
        const float x = (float)static_cast<const T*>(g.logits)[token * g.ld + first + j];
        const double k = x == -__builtin_inff() ? none : score64(g, x, most) / total + (g.bias ? (double)g.bias[first + j] : 0.0);
        two = fmax(two, fmin(one, k));
        one = fmax(one, k);
    }
    for (int off = 1; off < wide; off <<= 1) {
        const double a = __shfl_xor(one, off), b = __shfl_xor(two, off);
        two = fmax(fmax(two, b), fmin(one, a));
        one = fmax(one, a);
    }
    const double level = g.group_top == 2 && two != none ? level_of(one, two) : one;
    int better = 0;
    for (int o = 0; o < g.groups; ++o) {
        const double other = __shfl(level, o * wide + (threadIdx.x & 48));
        better += other > level || (other == level && o < mine);
    }
    kept = better < g.top_groups;
    return total;
}

// Four tokens' experts and weights, lane s of 16 those of slot s; `sure` is the row's.
template <class T, int V, bool SCORED>
__device__ __forceinline__ Choice route_four(const RouteView& g, const RouteLane<V>& l, int shift, const T* raw, int64_t token, bool& sure)
{
    const int lane = threadIdx.x & 15;
    const float none = -__builtin_inff();
    float key[V], most = none, total = 0.f;
    bool odd = l.bad, below = false;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        key[j] = (float)raw[j];
        odd |= !(key[j] < __builtin_inff());
        most = fmaxf(most, key[j]);
    }
    most = row_most(most);
    odd |= most == none;                                     // no expert at all
    float low, range, near, inv = 1.f;
    if (g.score == FOBQ_SOFTMAX && (SCORED || !g.renormalize)) {
#pragma unroll
        for (int j = 0; j < V; ++j) total += exp_of(key[j] - most);
        total = row_sum(total);
        inv = __builtin_amdgcn_rcpf(total);                  // the largest score
    }
    if constexpr (SCORED) {
        if (g.score == FOBQ_SOFTMAX) {
#pragma unroll
            for (int j = 0; j < V; ++j) key[j] = key[j] == none ? none : fmaf(exp_of(key[j] - most), inv, l.bias[j]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) key[j] = key[j] == none ? none : __builtin_amdgcn_rcpf(1.f + exp_of(-key[j])) + l.bias[j];
        }
        // A sigmoid is off by less than 8 units (exp2 and its argument, the sum, the reciprocal), a softmax by less than 32 of the largest (twenty additions more),
        // the sum with a bias by one unit of either: no more than half of `near` each.
        low = -l.most_bias;
        range = fmaf(2.f, l.most_bias, 1.01f * inv);
        near = 0x1p-24f * ((g.score == FOBQ_SOFTMAX ? 70.f : 20.f) * inv + 4.f * l.most_bias);
    } else {
        // (relative to the largest, so that the grid's offset is exact however far from 0 they are)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            below |= key[j] != none && !(key[j] - most >= -16.f);
            key[j] -= most;
        }
        low = -16.f;
        range = 16.f;
        near = 0.f;
    }
    // (the grid's offset is rounded, but the same for all; -Inf and what is below becomes step 0, which is no expert)
    const float unit = SCORED ? 8388600.f * __builtin_amdgcn_rcpf(range) : 8388600.f / 16.f, offset = fmaf(-low, unit, 2.f);
    const uint32_t behind = (15u - lane) << 4;
    uint32_t at[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float u = fmaf(key[j], unit, offset);
        at[j] = ((uint32_t)fmaxf(u, 0.f) << 8 | behind) | (15u - j);
    }
    if (g.groups > 1) {
        float first = none, second = none;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            second = fmaxf(second, fminf(first, key[j]));
            first = fmaxf(first, key[j]);
        }
        over_group(l.wide, [&](auto other) {
            const float f = other(first), s = other(second);
            second = fmaxf(fmaxf(second, s), fminf(first, f));
            first = fmaxf(first, f);
        });
        const bool two = SCORED && g.group_top == 2, real = l.mine < g.groups;
        bool kept = real;
        if (g.top_groups < g.groups) {
            // the same with the groups' words: the last one that is kept, and the first that is not
            const float level = two && second != none ? level_of(first, second) : first, half = two ? 0.5f : 1.f;
            const float u = fmaf(level, unit * half, offset);          // (for two, half the steps of a range twice as wide)
            const uint32_t word = real ? (uint32_t)fmaxf(u, 0.f) << 5 | (16u - l.mine) : 0u;
            uint32_t in = 0x80000000u;
            for (int i = 0; i < g.top_groups; ++i) in += row_most(word - in);
            const uint32_t out = row_most(word - in) + in;
            kept = word >= in;
            const bool close = out >> 5 != 0 && (in >> 5) - (out >> 5) <= (uint32_t)(2.f * near * unit * half) + 3u && !odd;
            if constexpr (SCORED) {
                if (__ballot(close)) {
                    bool other = kept;
                    route_row64<T, V>(g, l.first, l.there, l.mine, l.wide, token, most, true, other);
                    kept = close ? other : kept;
                }
            } else {
                odd |= close;
            }
        }
        if (!kept)
#pragma unroll
            for (int j = 0; j < V; ++j) at[j] &= 255u;
    }
    uint32_t last = 0x80000000u, mine = 0;
    for (int s = 0; s < g.top + 2; ++s) {
        uint32_t best = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) best = max(best, at[j] - last);
        last += row_most(best);
        if (lane == s) mine = last;
    }
    // the slot's expert and its logit
    const int index = 255 - (int)(mine & 255u), owner = index >> 4, group = owner >> shift;
    int expert = group * l.each + (owner - (group << shift)) * V + (index & 15);
    const bool have = mine > 255u && lane < g.top + 2 && !odd;
    float z = none, b = 0.f;
    if (have) {
        z = (float)static_cast<const T*>(g.logits)[token * g.ld + expert];
        if (SCORED && g.bias) b = g.bias[expert];
    }
    // Neighbours that the grid does not tell apart (of them those that are not equals: close); keys below the grid, or at its end, where it has too few.
    auto before = [](float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x111, 0xf, 0xf, true)); };
    const uint32_t ahead = (uint32_t)__builtin_amdgcn_mov_dpp((int)mine, 0x111, 0xf, 0xf, true) >> 8, step = (uint32_t)(near * unit) + 3u;
    const float z0 = before(z), b0 = before(b);
    const bool beside = have && lane > 0 && ahead - (mine >> 8) <= step;
    bool close = beside && !(z == z0 && b == b0);
    const int row0 = threadIdx.x & 48;
    const unsigned long long row = 0xffffull << row0, fell = __ballot(below), empty = __ballot(mine >> 8 <= 4u && lane <= g.top);
    const unsigned long long unsure = __ballot(close), both = 3ull << g.top << row0;
    const bool open = (__ballot(beside) & both) == both;
    if (__ballot(open)) {
        // Neither the last one chosen nor the next is apart from what follows, so that there may be larger ones behind the slots, also behind equals: the choice is
        // that of 64 bits only if all that is so near to the last one is its equal.
        const int from = row0 + g.top - 1;
        const float z1 = __shfl(z, from), b1 = __shfl(b, from);
        const int s1 = __shfl((int)(mine >> 8), from);
        bool other = false;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int s = (int)(at[j] >> 8);
            if (s > 0 && j < l.there && abs(s - s1) <= (int)step) other |= !((float)static_cast<const T*>(g.logits)[token * g.ld + l.first + j] == z1 && l.bias[j] == b1);
        }
        odd |= (__ballot(other) & row) != 0 && open;
    }
    if (unsure) {
        // The first top_k + 1 slots are put in order by 64 bits, which are all that are asked for if the last of them, or the next, is apart from the one before.
        if constexpr (SCORED) {
            bool other;
            const double total = g.score == FOBQ_SOFTMAX ? route_row64<T, V>(g, l.first, l.there, l.mine, l.wide, token, most, false, other) : 1.0;
            double k = have ? score64(g, z, most) / total + (double)b : -__builtin_inf();
            if (lane > g.top) k = -__builtin_inf();
            for (int i = 0; i <= g.top; ++i) {
                // neighbours in turn; a larger key, or the lower expert of two equal ones, goes first
                const int with = (threadIdx.x & 63) + ((lane + i) & 1 ? -1 : 1), to = with & 15;
                const bool pair = (with >> 4) == ((int)(threadIdx.x & 63) >> 4) && to <= g.top && lane <= g.top;
                const double k1 = __shfl(k, with);
                const int e1 = __shfl(expert, with);
                const float z1 = __shfl(z, with);
                const bool ahead1 = k1 > k || (k1 == k && (unsigned)e1 < (unsigned)expert);
                if (pair && k1 != -__builtin_inf() && k != -__builtin_inf() && ahead1 == (to > lane)) k = k1, expert = e1, z = z1;
            }
        } else {
            odd |= close;
        }
    }
    sure = (__ballot(odd) & row) == 0 && ((fell & row) == 0 || (empty & row) == 0);
    if (lane >= g.top || !have) z = none;
    const float p = route_weight(g, z, most, total, [](float x) { return row_most(x); }, [](float x) { return row_sum(x); });
    return Choice{z == none ? -1 : expert, z == none ? 0.f : g.scale * p};
}

template <class T, int V, bool SCORED>
__device__ __forceinline__ void route_tokens_by_four(RouteShared& sh, const RouteView& g, int64_t t0, int64_t t1)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), slot = lane & 15;
    sh.count[threadIdx.x] = 0;
    __syncthreads();
    auto keep = [&](int64_t token, int s, Choice c) {
        g.chosen[token * g.top + s] = c.expert;
        g.weights[token * g.top + s] = c.weight;
        sh.picked[(int)(token - t0) % 64 * g.top + s] = c.expert;
        if (c.expert >= 0) atomicAdd(&sh.count[c.expert], 1);
    };
    // 16 times four tokens of the wavefront; then those of them that it does again (bits of `again`: apart from the loop above, which needs its registers)
    for (int64_t start = t0 + 4 * wave; start < t1; start += 16 * 4 * ROUTE_WAVES) {
        uint64_t again = 0;
        {
            const RouteLane<V> l = route_lane<V, 16>(g);
            const int shift = __builtin_ctz(l.wide);
            for (int i = 0; i < 16; ++i) {
                const int64_t t = start + i * 4 * ROUTE_WAVES, token = min(t + lane / 16, t1 - 1);       // (rows behind the last token have that one)
                if (t >= t1) break;
                T raw[V];
                route_logits<T, V>(g, l, token, raw);
                bool sure;
                const Choice c = route_four<T, V, SCORED>(g, l, shift, raw, token, sure);
                const bool there = t + lane / 16 < t1;
                if (there && sure && slot < g.top) keep(token, slot, c);
                const unsigned long long undone = __ballot(there && !sure && slot == 0);
                again |= ((undone & 1) | (undone >> 15 & 2) | (undone >> 30 & 4) | (undone >> 45 & 8)) << (4 * i);
            }
        }
        constexpr int W = (V + 3) / 4;
        while (again) {
            const int i = __builtin_ctzll(again);
            again &= again - 1;
            const int64_t token = start + (i >> 2) * 4 * ROUTE_WAVES + (i & 3);
            const RouteLane<W> all = route_lane<W, 64>(g);
            T one[W];
            route_logits<T, W>(g, all, token, one);
            const Choice c = route_token<T, W, SCORED>(g, all, one);
            if (lane < g.top) keep(token, lane, c);
        }
    }
    __syncthreads();
}

// From the number of each expert's rows (count: of all tokens; before: of those in front of t0) where they lie; then those of tokens [t0, t1).  Every workgroup
// has the same starts; workgroup `part` of `parts` writes some of what is -1.  PICKED: the tokens' experts are in LDS already.
template <bool PICKED>
__device__ __forceinline__ void route_places(RouteShared& sh, const RouteView& g, int64_t t0, int64_t t1, int part, int parts)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t pairs = (int64_t)g.tokens * g.top;
    // thread e has expert e: an ascending sum over the threads
    const int mine = tid < g.experts ? sh.count[tid] : 0;
    int sum = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(sum, off);
        if (lane >= off) sum += v;
    }
    if (lane == 63) sh.sums[wave] = sum;
    __syncthreads();
    int at = sum - mine;
#pragma unroll
    for (int w = 0; w < ROUTE_WAVES; ++w) at += w < wave ? sh.sums[w] : 0;
    if (tid < g.experts) {
        sh.base[tid] = at + sh.before[tid];
        sh.seen[tid][0] = sh.seen[tid][1] = 0;
        if (part == 0) g.starts[tid] = at;
        if (tid == g.experts - 1) {
            sh.base[1024] = at + mine;
            if (part == 0) g.starts[g.experts] = at + mine;
        }
    }
    for (int64_t t = t0; t < t1; t += 64) {
        const int n = (int)min((int64_t)64, t1 - t) * g.top;
        __syncthreads();
        for (int i = tid; i < n; i += 64 * ROUTE_WAVES) {
            int e;
            if constexpr (PICKED) e = sh.picked[i];
            else e = sh.picked[i] = g.chosen[t * g.top + i];
            const int bit = (unsigned)i / (unsigned)g.top;
            if (e >= 0) atomicOr(&sh.seen[e][bit >> 5], 1u << (bit & 31));
        }
        __syncthreads();
        for (int i = tid; i < n; i += 64 * ROUTE_WAVES) {
            const int e = sh.picked[i], bit = (unsigned)i / (unsigned)g.top;
            int place = -1;
            if (e >= 0) {
                const uint32_t below = (1u << (bit & 31)) - 1;
                place = sh.base[e] + (bit < 32 ? __popc(sh.seen[e][0] & below) : __popc(sh.seen[e][0]) + __popc(sh.seen[e][1] & below));
                g.pairs[place] = (int)(t * g.top + i);
            }
            g.places[t * g.top + i] = place;
        }
        if (t + 64 < t1) {
            __syncthreads();
            if (tid < g.experts) {
                sh.base[tid] += __popc(sh.seen[tid][0]) + __popc(sh.seen[tid][1]);
                sh.seen[tid][0] = sh.seen[tid][1] = 0;
            }
        }
    }
    if (t0 >= t1) __syncthreads();
    for (int64_t i = sh.base[1024] + (int64_t)part * (64 * ROUTE_WAVES) + tid; i < pairs; i += (int64_t)parts * (64 * ROUTE_WAVES)) g.pairs[i] = -1;
}

// All of it where one workgroup has the tokens; otherwise the choice, and how often each expert is in it.  Bound by the vector instructions of the choice, not by memory:
// 16384 tokens x 256 fp32 logits take 16 to 20 us (17 MB, 4 us of a copy); alone, 64 tokens x 128 take 7.4 us, 64 x 256 with a bias and groups 12.8.  Of that, looking
// at equals beside the last choice is 0.3 to 1.5 us (16384 x 128, bf16, whose logits are often equal: 13.1 -> 14.1 with the places; in steps of 1/4: 13.6 -> 15.3).
// One workgroup for more than 64 tokens saves a launch (65 x 128: 9.9 -> 8.8) but has fewer wavefronts (128 x 128: 9.9 -> 11.7,
// 192 x 128: 10.2 -> 15.5): two launches from there on.
template <class T, int V, bool SCORED, bool FOUR>
__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_choose_kernel(RouteView g, RoutePlan p, int32_t* __restrict__ work)
{
    __shared__ RouteShared sh;
    const int64_t t0 = (int64_t)blockIdx.x * p.per_part, t1 = min((int64_t)g.tokens, t0 + p.per_part);
    const int tid = threadIdx.x;
    if (p.parts == 1) sh.before[tid] = 0;
    if constexpr (FOUR) route_tokens_by_four<T, V, SCORED>(sh, g, t0, t1);
    else route_tokens<T, V, SCORED>(sh, g, t0, t1);
    if (p.parts == 1) route_places<true>(sh, g, t0, t1, 0, 1);
    else if (tid < (g.experts + 3) / 4 * 4) work[(int64_t)blockIdx.x * ((g.experts + 3) / 4 * 4) + tid] = sh.count[tid];      // (rows of whole fours)
}

// Where the pairs lie: each workgroup sums the counts of all (256 x 256 whole numbers, from the L2) and ranks its own tokens' pairs.  16384 tokens x 8 of 256: 7 us.
__global__ __launch_bounds__(64 * ROUTE_WAVES) void route_places_kernel(RouteView g, RoutePlan p, const int32_t* __restrict__ work)
{
    __shared__ RouteShared sh;
    const int tid = threadIdx.x, part = blockIdx.x;
    const int64_t t0 = (int64_t)part * p.per_part, t1 = min((int64_t)g.tokens, t0 + p.per_part);
    // The counts of all parts, four neighbouring experts a thread; the threads that have the same four deal the parts among them.
    sh.count[tid] = sh.before[tid] = 0;
    __syncthreads();
    typedef int i4 __attribute__((ext_vector_type(4)));
    const int quads = (g.experts + 3) / 4, quad = tid % quads, share = 64 * ROUTE_WAVES / quads, first = tid / quads;
    if (first < share) {
        const i4* __restrict__ row = reinterpret_cast<const i4*>(work) + quad;
        i4 before = {0, 0, 0, 0}, behind = {0, 0, 0, 0};
        int w = first;
#pragma unroll 8
        for (; w < part; w += share) before += row[(int64_t)w * quads];
#pragma unroll 8
        for (; w < p.parts; w += share) behind += row[(int64_t)w * quads];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * quad + i < g.experts) {
                atomicAdd(&sh.count[4 * quad + i], before[i] + behind[i]);
                atomicAdd(&sh.before[4 * quad + i], before[i]);
            }
    }
    __syncthreads();
    route_places<false>(sh, g, t0, t1, part, p.parts);
}

// LANES lanes have 8 LANES columns of a token, its rows four at a time under way.  (32768 rows of 4096 bf16 to 8192 tokens with a base: 90 us, 4.5 TB/s.)
template <class T, int LANES>
__global__ __launch_bounds__(256) void expert_sum_kernel(ExpertSum g, unsigned across)
{
    constexpr int AT_ONCE = 4;
    const int lane = threadIdx.x & (LANES - 1);
    int64_t item = (int64_t)blockIdx.x * (256 / LANES) + (threadIdx.x / LANES);
    if constexpr (LANES == 64) item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t token = across == 1 ? item : item / across;
    if (token >= g.tokens) return;
    const int64_t col = (item - token * across) * (8 * LANES) + 8 * lane;
    const int left = (int)min((int64_t)8, g.cols - col);
    if (left <= 0) return;
    const T* y = static_cast<const T*>(g.y) + col;
    auto load = [&](const T* p, T* x) {
        if (left == 8) __builtin_memcpy(x, p, 8 * sizeof(T));
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = i < left ? p[i] : (T)0.f;
        }
    };
    T first[8];
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (g.base) load(static_cast<const T*>(g.base) + token * g.base_ld + col, first);
    for (int s0 = 0; s0 < g.top; s0 += AT_ONCE) {
        T x[AT_ONCE][8];
        float w[AT_ONCE];
        bool there[AT_ONCE];
#pragma unroll
        for (int s = 0; s < AT_ONCE; ++s) {
            const int64_t slot = token * g.top + min(s0 + s, g.top - 1);
            const int place = g.places[slot];
            w[s] = g.weights[slot];
            there[s] = s0 + s < g.top && (unsigned)place < (unsigned)g.rows;
            if (there[s]) load(y + (int64_t)place * g.ld, x[s]);
        }
        if (s0 == 0 && g.base) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = (float)first[i];
        }
#pragma unroll
        for (int s = 0; s < AT_ONCE; ++s)
            if (there[s]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = fmaf(w[s], (float)x[s][i], sum[i]);
            }
    }
    T* out = static_cast<T*>(g.out) + token * g.out_ld + col;
    if (left == 8) store8(out, sum);
    else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) out[i] = (T)sum[i];
    }
}

RoutePlan route_plan(int64_t tokens)
{
    const int64_t per = std::max<int64_t>(1, (tokens + 64 * 256 - 1) / (64 * 256)) * 64;
    return RoutePlan{(int)std::max<int64_t>(1, (tokens + per - 1) / per), (int)per};
}

int64_t route_workspace(const RoutePlan& p, int experts) { return p.parts > 1 ? (int64_t)p.parts * ((experts + 3) / 4 * 4) * (int64_t)sizeof(int32_t) : 0; }

// experts of a lane where a token has `lanes`
static int route_each(const RouteView& g, int lanes)
{
    if (g.groups > lanes) return 1 << 30;
    int wide = lanes;
    while (wide * g.groups > lanes) wide >>= 1;
    return (g.experts / g.groups + wide - 1) / wide;
}

template <class T, int V, bool FOUR>
static void choose_of(hipStream_t s, const RoutePlan& p, const RouteView& g, int32_t* work)
{
    const dim3 grid((unsigned)p.parts), block(64 * ROUTE_WAVES);
    if (g.bias || (g.groups > 1 && g.group_top == 2)) hipLaunchKernelGGL((route_choose_kernel<T, V, true, FOUR>), grid, block, 0, s, g, p, work);
    else hipLaunchKernelGGL((route_choose_kernel<T, V, false, FOUR>), grid, block, 0, s, g, p, work);
}

template <class T>
static hipError_t route_of(hipStream_t s, const RoutePlan& p, const RouteView& g, int32_t* work)
{
    const int four = route_each(g, 16), each = route_each(g, 64);
    if (four <= 16 && g.top <= ROW_TOP) {
        if (four <= 1) choose_of<T, 1, true>(s, p, g, work);
        else if (four <= 2) choose_of<T, 2, true>(s, p, g, work);
        else if (four <= 4) choose_of<T, 4, true>(s, p, g, work);
        else if (four <= 8) choose_of<T, 8, true>(s, p, g, work);
        else choose_of<T, 16, true>(s, p, g, work);
    } else if (each <= 1) choose_of<T, 1, false>(s, p, g, work);
    else if (each <= 2) choose_of<T, 2, false>(s, p, g, work);
    else if (each <= 4) choose_of<T, 4, false>(s, p, g, work);
    else if (each <= 8) choose_of<T, 8, false>(s, p, g, work);
    else if (each <= 16) choose_of<T, 16, false>(s, p, g, work);
    else choose_of<T, 32, false>(s, p, g, work);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL(route_places_kernel, dim3((unsigned)p.parts), dim3(64 * ROUTE_WAVES), 0, s, g, p, work);
    return hipGetLastError();
}

hipError_t launch_route(hipStream_t s, const RoutePlan& p, const RouteView& g, int type, int32_t* work)
{
    if (type == FOBQ_F32) return route_of<float>(s, p, g, work);
    return type == FOBQ_BF16 ? route_of<bf16_t>(s, p, g, work) : route_of<f16_t>(s, p, g, work);
}

template <class T, int LANES>
static hipError_t sum_by(hipStream_t s, const ExpertSum& g)
{
    const unsigned across = (unsigned)((g.cols + 8 * LANES - 1) / (8 * LANES)), per = 256 / LANES;
    hipLaunchKernelGGL((expert_sum_kernel<T, LANES>), dim3((unsigned)(((int64_t)g.tokens * across + per - 1) / per)), dim3(256), 0, s, g, across);
    return hipGetLastError();
}

template <class T>
static hipError_t sum_of(hipStream_t s, const ExpertSum& g)
{
    if (g.cols <= 64) return sum_by<T, 8>(s, g);
    if (g.cols <= 128) return sum_by<T, 16>(s, g);
    return g.cols <= 256 ? sum_by<T, 32>(s, g) : sum_by<T, 64>(s, g);
}

hipError_t launch_expert_sum(hipStream_t s, const ExpertSum& g, int type)
{
    if (type == FOBQ_F32) return sum_of<float>(s, g);
    return type == FOBQ_BF16 ? sum_of<bf16_t>(s, g) : sum_of<f16_t>(s, g);
}

}  // namespace fobq
