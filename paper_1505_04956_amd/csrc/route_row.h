// A row of logits to the experts with the best keys and their weights, by one wave.
#pragma once

#include <type_traits>

#include "experts_internal.h"

namespace asgd {

namespace {

constexpr float OUT = -INFINITY;          // key of an expert that cannot be chosen

// V consecutive elements of a row from e on, of which those before E exist
template <class Ty, int V> struct Lane { typename Ty::T v[V]; };
template <class Ty, int V> __device__ __forceinline__ Lane<Ty, V> load_lane(const typename Ty::T *row, int e, int E, bool wide)
{
    Lane<Ty, V> r;
    constexpr int BYTES = V * sizeof(typename Ty::T), N = BYTES < 16 ? BYTES : 16;
    if (wide) {
        if (e < E)
#pragma unroll
            for (int i = 0; i < BYTES / N; i++) {
                if constexpr (N == 16) *((uint4 *)r.v + i) = *((const uint4 *)(row + e) + i);
                else if constexpr (N == 8) *(uint2 *)r.v = *(const uint2 *)(row + e);
                else if constexpr (N == 4) *(uint32_t *)r.v = *(const uint32_t *)(row + e);
                else r.v[0] = row[e];
            }
    } else
#pragma unroll
        for (int i = 0; i < V; i++)
            if (e + i < E) r.v[i] = row[e + i];
    return r;
}
template <class Ty, int V> bool rows_of_lanes(const void *p, int64_t stride, int E)
{
    constexpr int BYTES = V * sizeof(typename Ty::T), N = BYTES < 16 ? BYTES : 16;
    return E % V == 0 && (uintptr_t)p % N == 0 && stride * (int64_t)sizeof(typename Ty::T) % N == 0;
}

// l of the lane's experts (out: -infinity), and whether an expert that is in has something that is not a number
template <class Ty, int V>
__device__ __forceinline__ bool logits_of(const Lane<Ty, V> &r, const float (&bias)[V], int E, int lane, float (&l)[V])
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < V; i++) {
        l[i] = lane * V + i < E && bias[i] != OUT ? (float)r.v[i] : OUT;
        bad |= (l[i] != l[i]) | ((l[i] != OUT) & (bias[i] != bias[i]));
    }
    return __any(bad);
}
template <int V> __device__ __forceinline__ void load_bias(const float *bias, int E, int lane, float (&b)[V])
{
#pragma unroll
    for (int i = 0; i < V; i++) b[i] = bias && lane * V + i < E ? bias[lane * V + i] : 0.0f;
}

// 1 / (1 + exp(-l)), in the operations of the definition
__device__ __forceinline__ float sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }

// an order among numbers: what is not one comes last of those that are in
__device__ __forceinline__ float as_key(float v) { return v == v ? v : -3.402823466e38f; }

template <class T, int V> __device__ __forceinline__ T lane_best(const T (&v)[V])
{
    T m = v[0];
#pragma unroll
    for (int i = 1; i < V; i++) m = max(m, v[i]);
    return m;
}

// the two best of two pairs of two best
__device__ __forceinline__ void join_best(float &m1, float &m2, float o1, float o2)
{
    m2 = fmaxf(fmaxf(m2, o2), fminf(m1, o1));
    m1 = fmaxf(m1, o1);
}

template <class Ty, int V, bool SORTED> __device__ __forceinline__ void route_row(const RouteArgs &a, int64_t t, int lane, const Lane<Ty, V> &raw, const float (&bias)[V])
{
    const typename Ty::T *row = (const typename Ty::T *)a.logits + t * a.stride;
    const int E = a.E, k = a.rule.k;
    const bool soft = a.rule.score == ASGD_SCORE_SOFTMAX;
    float l[V], key[V];
    const bool bad = logits_of<Ty, V>(raw, bias, E, lane, l);
    float top = 0.0f, total = 1.0f;
    if (soft && (!a.rule.renormalize || a.bias || (a.rule.groups > 1 && a.rule.group_by == ASGD_GROUP_BEST_TWO))) {
        top = wave_max(lane_best(l));
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < V; i++) sum += l[i] == OUT ? 0.0f : expf(l[i] - top);
        total = wave_sum(sum);
    }
    const bool two = a.rule.groups > 1 && a.rule.group_by == ASGD_GROUP_BEST_TWO;
    float score[V];
    if (a.bias || two) {
        if (soft)
#pragma unroll
            for (int i = 0; i < V; i++) score[i] = expf(l[i] - top) / total;
        else
#pragma unroll
            for (int i = 0; i < V; i++) score[i] = sigmoid(l[i]);
#pragma unroll
        for (int i = 0; i < V; i++) score[i] = l[i] == OUT ? OUT : as_key(score[i] + bias[i]);       // (no bias: plus zero)
    }
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < V; i++) key[i] = score[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; i++) key[i] = as_key(l[i]);
    }
    if (a.rule.groups > 1) {
        const int G = a.rule.groups, width = E / G, lanes = width / V;
        const auto by = [&](int i) { return two ? score[i] : key[i]; };
        unsigned long long stays = 0;
        if (lanes * V == width && lanes <= 16 && (lanes & (lanes - 1)) == 0) {
            // a group is 1, 2, .. 16 whole lanes next to each other: all groups at once
            float m1 = OUT, m2 = OUT;
#pragma unroll
            for (int i = 0; i < V; i++) join_best(m1, m2, by(i), OUT);
            if (lanes > 1) join_best(m1, m2, across<XOR1>(m1), across<XOR1>(m2));
            if (lanes > 2) join_best(m1, m2, across<XOR2>(m1), across<XOR2>(m2));
            if (lanes > 4) join_best(m1, m2, across<MIRROR8>(m1), across<MIRROR8>(m2));
            if (lanes > 8) join_best(m1, m2, across<MIRROR16>(m1), across<MIRROR16>(m2));
            const float mine = two ? as_key(m1 + m2) : m1;
            const int g = lane / lanes;
            int before = 0;                                                   // groups that are taken before the lane's
            for (int o = 0; o < G; o++) {
                const float other = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), o * lanes));
                before += other > mine || (other == mine && o < g) ? 1 : 0;
            }
#pragma unroll
            for (int i = 0; i < V; i++)
                if (before >= a.rule.kept) key[i] = OUT;
        } else {
            float mine = OUT;                                                 // lane g: how group g is judged
            for (int g = 0; g < G; g++) {
                float m1 = OUT, m2 = OUT;                                     // the lane's two best of the group
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const int e = lane * V + i;
                    if (e >= g * width && e < (g + 1) * width) join_best(m1, m2, by(i), OUT);
                }
                const float best = wave_max(m1);
                float judged = best;
                if (two) {
                    // the second best: the lowest lane with the best gives that one up
                    const unsigned long long has = __ballot(m1 == best);
                    const bool gives = lane == __ffsll((long long)has) - 1;
                    judged = as_key(best + wave_max(gives ? m2 : m1));
                }
                if (lane == g) mine = judged;
            }
            unsigned long long open = G == 64 ? ~0ull : (1ull << G) - 1;
            for (int n = 0; n < a.rule.kept; n++) {
                const bool here = open >> lane & 1;
                const float best = wave_max(here ? mine : OUT);
                const int g = __ffsll((long long)__ballot(here && mine == best)) - 1;
                open &= ~(1ull << g);
                stays |= 1ull << g;
            }
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int e = lane * V + i;
                if (e < E && !(stays >> (e / width) & 1)) key[i] = OUT;
            }
        }
    }
    int id = -1;                                                              // lane j: choice j
    const int none = as_integer(OUT);
    int order[V];
#pragma unroll
    for (int i = 0; i < V; i++) order[i] = as_integer(key[i] + 0.0f);
    // SORTED: a lane's experts are put in order first (largest key first, of equal ones the lower index): its first is then all that can be
    // chosen next, and the lane that it is chosen from gives it up.  Else a choice is looked for among all V again.
    uint64_t places = 0;                                                      // four bits each, in that order
    if constexpr (SORTED) {
        int at[V];
#pragma unroll
        for (int i = 0; i < V; i++) at[i] = i;
#pragma unroll
        for (int i = 1; i < V; i++)
#pragma unroll
            for (int n = i; n > 0; n--) {
                const bool swap = order[n] > order[n - 1];
                const int u = order[n], w = order[n - 1];
                const int p = at[n], q = at[n - 1];
                order[n] = swap ? w : u;
                order[n - 1] = swap ? u : w;
                at[n] = swap ? q : p;
                at[n - 1] = swap ? p : q;
            }
#pragma unroll
        for (int i = 0; i < V; i++) places |= (uint64_t)at[i] << 4 * i;
    }
    for (int j = 0; j < k; j++) {
        const int m = SORTED ? order[0] : lane_best(order), best = wave_max(m);
        if (best == none) break;
        const int owner = __ffsll((long long)__ballot(m == best)) - 1;
        const bool mine = lane == owner;
        int place;
        if constexpr (SORTED) {
            place = __builtin_amdgcn_readlane((int)(uint32_t)places, owner) & 15;
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int now = order[i], then = i + 1 < V ? order[i + 1 < V ? i + 1 : i] : none;
                order[i] = mine ? then : now;
            }
            places = mine ? places >> 4 : places;
        } else {
            unsigned has = 0;
#pragma unroll
            for (int i = 0; i < V; i++) has |= (unsigned)(__ballot(order[i] == best) >> owner & 1) << i;
            place = __ffs(has) - 1;
#pragma unroll
            for (int i = 0; i < V; i++)
                if (mine && i == place) order[i] = none;
        }
        if (lane == j) id = owner * V + place;
    }
    const float chosen = id >= 0 ? (float)row[id] : OUT;
    float share;
    if (soft && a.rule.renormalize) {                                         // (all lanes or none)
        const float largest = wave_max(chosen);
        share = expf(chosen - largest);
    } else share = soft ? expf(chosen - top) / total : sigmoid(chosen);
    if (chosen == OUT) share = 0.0f;
    if (a.rule.renormalize) {
        const float sum = wave_sum(share);
        share = sum > 0.0f ? share / sum : sum == 0.0f ? 0.0f : sum;
    }
    if (lane < k) {
        a.ids[t * k + lane] = id;
        a.weights[t * k + lane] = bad && id >= 0 ? __uint_as_float(0x7FC00000u) : share * a.rule.scale;
    }
}

template <class F> hipError_t with_width(int E, F f)
{
    if (E <= 64) return f(std::integral_constant<int, 1>{});
    if (E <= 128) return f(std::integral_constant<int, 2>{});
    if (E <= 256) return f(std::integral_constant<int, 4>{});
    if (E <= 512) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

}  // namespace

}  // namespace asgd
