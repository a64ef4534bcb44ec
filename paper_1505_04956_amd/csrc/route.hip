// Routing of rows to experts: scores, the best k by key, their weights; the gradient of the logits; the order by expert.
//
// One wave takes a row after the other.  Lane i holds the V consecutive experts i * V .. i * V + V - 1, so that among equal keys
// the lowest lane, and in it the lowest register, is the lowest index.  The row is read once, and what bounds it is vector instructions, nine of
// ten cycles: a score is some 27 of them (exp and a division, both rounded as the definition has them), a choice 18 (a maximum over lanes,
// six, whose lane a ballot finds and which that lane then gives up).  65536 rows of 256 in float32, eight chosen by sigmoid, bias and groups:
// 69 us (1.0 TB/s); 8 of 256 by softmax without a bias, 41 us; one row of 64, 2.6 us.
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

template <class Ty, int V, bool SORTED> __global__ __launch_bounds__(256) void route_kernel(RouteArgs a, bool wide)
{
    const int lane = threadIdx.x & 63;
    const int64_t step = (int64_t)gridDim.x * 4;
    int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    const typename Ty::T *logits = (const typename Ty::T *)a.logits;
    Lane<Ty, V> next = load_lane<Ty, V>(logits + t * a.stride, lane * V, a.E, wide);
    float bias[V];
    load_bias<V>(a.bias, a.E, lane, bias);
    for (; t < a.T; t += step) {
        const Lane<Ty, V> now = next;
        if (t + step < a.T) next = load_lane<Ty, V>(logits + (t + step) * a.stride, lane * V, a.E, wide);
        route_row<Ty, V, SORTED>(a, t, lane, now, bias);
    }
}

// With the choice held fixed: w_j = c s_j or c s_j / sum of the chosen s.
//   g_j = c dw_j                      or  (c / sum) (dw_j - sum_i dw_i s_i / sum)
//   sigmoid: dl_j = g_j s_j (1 - s_j);  softmax: dl_e = s_e (g_e - sum_i g_i s_i), whose inner sum is 0 when renormalised
// Both differences stay what they are when all dw, or all g, are lessened by the same number, since the shares they are weighed by add up to
// one.  That number is the one of the largest share: next to a share of one its own difference would cancel, and the gradient of a confident
// router with it.
// The k gradients are scattered over a row in the LDS and leave as whole lines.  Memory bounds it: 65536 rows of 256 in float32 take 29 us, 4.9
// TB/s of logits read and gradients written, what a large copy reaches.
template <class Ty, int V>
__device__ __forceinline__ void route_row_backward(const RouteArgs &a, int64_t t, int lane, float *mine, const Lane<Ty, V> &raw, const float (&bias)[V], bool wide)
{
    typedef typename Ty::T T;
    const T *row = (const T *)a.logits + t * a.stride;
    T *out = (T *)a.d_logits + t * a.d_stride;
    const int E = a.E, k = a.rule.k;
    const bool soft = a.rule.score == ASGD_SCORE_SOFTMAX, renorm = a.rule.renormalize;
    int id = lane < k ? a.ids_in[t * k + lane] : -1;
    if (id >= E) id = -1;
    const bool there = id >= 0;
    const float chosen = there ? (float)row[id] : OUT;
    const float dw = there ? a.d_weights[t * k + lane] : 0.0f;
    const auto fill = [&](float v) {
#pragma unroll
        for (int i = 0; i < V; i++) mine[i * 64 + lane] = v;
    };
    if (!soft || renorm) fill(0.0f);
    float l[V];
    const bool bad = logits_of<Ty, V>(raw, bias, E, lane, l);
    float top = 0.0f, total = 1.0f, score[V];
    if (soft && !renorm) {
        top = wave_max(lane_best(l));
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < V; i++) sum += score[i] = l[i] == OUT ? 0.0f : expf(l[i] - top);
        total = wave_sum(sum);
#pragma unroll
        for (int i = 0; i < V; i++) score[i] = l[i] == OUT ? 0.0f : score[i] / total;
    }
    float share;
    const float largest = wave_max(chosen);
    if (soft && renorm) share = there ? expf(chosen - largest) : 0.0f;
    else share = !there ? 0.0f : soft ? expf(chosen - top) / total : sigmoid(chosen);
    const float rest = soft ? 0.0f : sigmoid(-chosen);         // 1 - s of a sigmoid (not by that difference, which loses a confident expert's gradient)
    const auto of_first = [&](bool which, float v) {           // v of the first such lane, 0 without any
        const unsigned long long has = __ballot(which);
        return has ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), __ffsll((long long)has) - 1)) : 0.0f;
    };
    float g, grad;
    if (renorm) {
        const float sum = wave_sum(share);
        const float part = sum == 0.0f ? 0.0f : share / sum;
        const float off = dw - of_first(there && chosen == largest, dw);
        g = a.rule.scale * (off - wave_sum(off * part));
        if (sum == 0.0f) g = 0.0f;
        grad = soft ? g * part : g * part * rest;              // (and not g / sum * share, beyond 32 bits where scores are small)
    } else {
        const float base = soft ? of_first(there && chosen == top, dw) : 0.0f;
        if (soft) fill(-a.rule.scale * base);                                 // (an expert that is not chosen: dw = 0)
        g = a.rule.scale * (dw - base);
        grad = soft ? g : g * share * rest;
    }
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
    if (there) mine[id] = grad;
    __builtin_amdgcn_wave_barrier();
    __threadfence_block();
    float d[V], inner = 0.0f;
#pragma unroll
    for (int i = 0; i < V; i++) d[i] = mine[lane * V + i];
    if (soft && !renorm) {
#pragma unroll
        for (int i = 0; i < V; i++) inner = fmaf(score[i], d[i], inner);
        inner = wave_sum(inner);
#pragma unroll
        for (int i = 0; i < V; i++) d[i] = l[i] == OUT ? 0.0f : score[i] * (d[i] - inner);
    }
    T u[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        float v = d[i];
        if (bad && l[i] != OUT) v = __uint_as_float(0x7FC00000u);
        u[i] = (T)v;
    }
    if (wide) {
        constexpr int BYTES = V * sizeof(T), N = BYTES < 16 ? BYTES : 16;
        if (lane * V < E)
#pragma unroll
            for (int i = 0; i < BYTES / N; i++) {
                if constexpr (N == 16) *((uint4 *)(out + lane * V) + i) = *((uint4 *)u + i);
                else if constexpr (N == 8) *(uint2 *)(out + lane * V) = *(uint2 *)u;
                else if constexpr (N == 4) *(uint32_t *)(out + lane * V) = *(uint32_t *)u;
                else out[lane] = u[0];
            }
    } else
#pragma unroll
        for (int i = 0; i < V; i++)
            if (lane * V + i < E) out[lane * V + i] = u[i];
    __builtin_amdgcn_wave_barrier();
}

template <class Ty, int V> __global__ __launch_bounds__(256) void route_backward_kernel(RouteArgs a, bool wide, bool wide_out)
{
    __shared__ float grads[4][64 * V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t step = (int64_t)gridDim.x * 4;
    int64_t t = (int64_t)blockIdx.x * 4 + wave;
    if (t >= a.T) return;
    const typename Ty::T *logits = (const typename Ty::T *)a.logits;
    Lane<Ty, V> next = load_lane<Ty, V>(logits + t * a.stride, lane * V, a.E, wide);
    float bias[V];
    load_bias<V>(a.bias, a.E, lane, bias);
    for (; t < a.T; t += step) {
        const Lane<Ty, V> now = next;
        if (t + step < a.T) next = load_lane<Ty, V>(logits + (t + step) * a.stride, lane * V, a.E, wide);
        route_row_backward<Ty, V>(a, t, lane, grads[wave], now, bias, wide_out);
    }
}

// ---- the order by expert --------------------------------------------------------------------------------------------
// A counting sort that keeps the order of slots.  Lanes that have the same expert find each other by the bits of its number, and each
// learns how many lower lanes have it.  A workgroup takes 4096 slots at a time, 256 a wave, whose ids it holds in registers:
// counts of each wave, sums over the waves, places.  Where there are more slots, chunks of them are counted first, and every
// workgroup adds up for itself what lies before its chunk.  Steps that wait for each other bound it, not data: 120 slots of 100 experts take 7.4
// us, 16372 of 64 take 5.8 (counts) and 11 us (places), 524288 of 256 both together 25 us.
constexpr int HELD = 4, WAVE_SLOTS = 64 * HELD, BLOCK_SLOTS = 16 * WAVE_SLOTS, MOST_CHUNKS = 256;

__device__ __forceinline__ unsigned long long same_expert(int e, int bits)
{
    unsigned long long same = ~0ull;
    for (int bit = 0; bit < bits; bit++) {
        const unsigned long long set = __ballot(e >> bit & 1);
        same &= e >> bit & 1 ? set : ~set;
    }
    return same;
}

// a wave's ids from `begin` on; E: none
__device__ __forceinline__ void load_ids(const int32_t *ids, int64_t begin, int64_t end, int E, int (&e)[HELD])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int r = 0; r < HELD; r++) {
        const int64_t s = begin + r * 64 + lane;
        e[r] = s < end ? ids[s] : -1;
    }
#pragma unroll
    for (int r = 0; r < HELD; r++) e[r] = (unsigned)e[r] < (unsigned)E ? e[r] : E;
}

// Exclusive sums over the experts of their counts and of their blocks of 128, by one workgroup of 1024 (thread e has expert e).
__device__ int sum_experts(int n, int E, int32_t *offsets, int32_t *blocks, bool write)
{
    __shared__ int part[2][16];
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    const int v0 = e < E ? n : 0, v1 = e < E ? (n + BLOCK8 - 1) / BLOCK8 : 0;
    int s0 = v0, s1 = v1;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int u0 = __shfl_up(s0, m), u1 = __shfl_up(s1, m);
        if (lane >= m) { s0 += u0; s1 += u1; }
    }
    if (lane == 63) { part[0][wave] = s0; part[1][wave] = s1; }
    __syncthreads();
    int b0 = 0, b1 = 0;
    for (int w = 0; w < wave; w++) { b0 += part[0][w]; b1 += part[1][w]; }
    if (write) {
        if (e < E) { offsets[e] = b0 + s0 - v0; blocks[e] = b1 + s1 - v1; }
        if (e == E - 1) { offsets[E] = b0 + s0; blocks[E] = b1 + s1; }
    }
    return b0 + s0 - v0;
}

// table[chunk][e]: the slots of expert e in a chunk of `chunk` slots
__global__ __launch_bounds__(1024) void plan_count_kernel(const int32_t *ids, int64_t slots, int64_t chunk, int E, int bits, int *table)
{
    __shared__ int count[ASGD_ROUTE_MAX_EXPERTS + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i <= E; i += 1024) count[i] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * chunk, end = begin + chunk < slots ? begin + chunk : slots;
    for (int64_t s = begin + wave * WAVE_SLOTS; s < end; s += BLOCK_SLOTS) {
        int e[HELD];
        load_ids(ids, s, end, E, e);
#pragma unroll
        for (int r = 0; r < HELD; r++) {
            const unsigned long long same = same_expert(e[r], bits);
            if (!(same & ((1ull << lane) - 1))) atomicAdd(&count[e[r]], __popcll(same));      // (whole numbers: any order gives the same)
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < E; i += 1024) table[(int64_t)blockIdx.x * E + i] = count[i];
}

// chunks = 1: no table
__global__ __launch_bounds__(1024) void plan_place_kernel(const int32_t *ids, asgd_route_order o, int64_t chunk, int chunks, int bits, const int *table)
{
    extern __shared__ unsigned short ranks[];       // [16][E + 1]: of a wave, then slots of the expert in the waves before it
    __shared__ int next[ASGD_ROUTE_MAX_EXPERTS], total[ASGD_ROUTE_MAX_EXPERTS];
    __shared__ int used;
    const int E = o.E, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, me = threadIdx.x;
    const int64_t slots = o.T * o.k, begin = blockIdx.x * chunk, end = begin + chunk < slots ? begin + chunk : slots;
    unsigned short *mine = ranks + wave * (E + 1);
    const int waves = end - begin >= BLOCK_SLOTS ? 16 : (int)((end - begin + WAVE_SLOTS - 1) / WAVE_SLOTS);       // that have slots
    int e[HELD];
    const auto count = [&](int64_t s) {
        if (wave < waves) {
            for (int i = lane; i <= E; i += 64) mine[i] = 0;
            __threadfence_block();
            load_ids(ids, s + wave * WAVE_SLOTS, end, E, e);
#pragma unroll
            for (int r = 0; r < HELD; r++) {
                const unsigned long long same = same_expert(e[r], bits);
                if (!(same & ((1ull << lane) - 1))) mine[e[r]] += (unsigned short)__popcll(same);
                __builtin_amdgcn_wave_barrier();
                __threadfence_block();
            }
        }
        __syncthreads();
    };
    if (chunks > 1) {
        // what all chunks have, and those before this one: the threads of an expert take a part of the chunks each
        if (me < E) next[me] = total[me] = 0;
        __syncthreads();
        const int parts = 1024 / E, part = me / E, mine_e = me - part * E;
        int all = 0, before = 0;
        if (part < parts)
            for (int c = part; c < chunks; c += parts) {
                const int n = table[(int64_t)c * E + mine_e];
                all += n;
                before += c < (int)blockIdx.x ? n : 0;
            }
        if (part < parts) {
            atomicAdd(&total[mine_e], all);
            atomicAdd(&next[mine_e], before);
        }
        __syncthreads();
    } else {
        count(begin);
        if (me < E) {
            int n = 0;
            for (int w = 0; w < waves; w++) n += ranks[w * (E + 1) + me];
            total[me] = n;
            next[me] = 0;
        }
        __syncthreads();
    }
    const int n = me < E ? total[me] : 0, offset = sum_experts(n, E, o.offsets, o.blocks, blockIdx.x == 0);
    if (me < E) next[me] += offset;
    if (me == E - 1) used = offset + n;
    __syncthreads();
    for (int64_t s = begin; s < end; s += BLOCK_SLOTS) {
        if (chunks > 1) count(s);
        int sum = 0;
        if (me < E)
            for (int w = 0; w < waves; w++) {
                const int m = ranks[w * (E + 1) + me];
                ranks[w * (E + 1) + me] = (unsigned short)sum;
                sum += m;
            }
        __syncthreads();
        if (wave < waves)
#pragma unroll
            for (int r = 0; r < HELD; r++) {
                const int64_t slot = s + wave * WAVE_SLOTS + r * 64 + lane;
                const unsigned long long same = same_expert(e[r], bits), before = same & ((1ull << lane) - 1);
                const bool there = e[r] < E;
                int rank = 0;
                if (there) rank = mine[e[r]] + __popcll(before);
                __builtin_amdgcn_wave_barrier();
                __threadfence_block();
                if (there && !before) mine[e[r]] = (unsigned short)(rank + __popcll(same));
                __builtin_amdgcn_wave_barrier();
                __threadfence_block();
                if (slot < end) {
                    const int place = there ? next[e[r]] + rank : -1;
                    o.places[slot] = place;
                    if (there) o.slots[place] = (int32_t)slot;
                }
            }
        __syncthreads();
        if (me < E) next[me] += sum;
        __syncthreads();
    }
    for (int64_t p = begin + me; p < end; p += 1024)
        if (p >= used) o.slots[p] = -1;
}

// slots of a chunk: one workgroup's where that gives few chunks
int64_t plan_chunk(int64_t slots) { return BLOCK_SLOTS * ((slots + (int64_t)BLOCK_SLOTS * MOST_CHUNKS - 1) / ((int64_t)BLOCK_SLOTS * MOST_CHUNKS)); }

template <class F> hipError_t with_width(int E, F f)
{
    if (E <= 64) return f(std::integral_constant<int, 1>{});
    if (E <= 128) return f(std::integral_constant<int, 2>{});
    if (E <= 256) return f(std::integral_constant<int, 4>{});
    if (E <= 512) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

}  // namespace

// four waves a workgroup, eight workgroups a compute unit; a wave's next row is on its way while it works on one
static unsigned route_grid(int64_t T) { return (unsigned)((T + 3) / 4 < 2048 ? (T + 3) / 4 : 2048); }

// In order or not, us of float32 softmax over 65536 rows (512: 32768, 1024: 16384) for 1, 2, 4, 8 choices:
//    64   16.4 18.0 21.9 29.6   not   16.9 18.8 23.2 32.4
//   128   19.4 21.4 26.1 35.2   not   19.4 22.2 28.1 39.9
//   256   23.7 26.1 30.8 41.0   not   22.7 26.7 35.1 53.7
//   512   25.3 26.9 30.1 36.5   not   19.3 22.3 29.5 45.2
//  1024   25.5 26.7 29.3 33.8   not   22.1 25.8 33.5 48.7
// The rule, fewer than four choices of more than 256 experts without order, is not the better of the two by 1 us for one choice of 256
// (which would be a kernel more for each type) and by 0.6 for four of 512.
hipError_t launch_route(const RouteArgs &a, int type, hipStream_t s)
{
    const unsigned grid = route_grid(a.T);
    return with_type(type, [&](auto ty) {
        return with_width(a.E, [&](auto v) {
            constexpr int V = decltype(v)::value;
            const bool wide = rows_of_lanes<decltype(ty), V>(a.logits, a.stride, a.E);
            if constexpr (V >= 8)
                if (a.rule.k < 4) {
                    route_kernel<decltype(ty), V, false><<<grid, 256, 0, s>>>(a, wide);
                    return hipGetLastError();
                }
            route_kernel<decltype(ty), V, true><<<grid, 256, 0, s>>>(a, wide);
            return hipGetLastError();
        });
    });
}

hipError_t launch_route_backward(const RouteArgs &a, int type, hipStream_t s)
{
    const unsigned grid = route_grid(a.T);
    return with_type(type, [&](auto ty) {
        return with_width(a.E, [&](auto v) {
            route_backward_kernel<decltype(ty), decltype(v)::value><<<grid, 256, 0, s>>>(a, rows_of_lanes<decltype(ty), decltype(v)::value>(a.logits, a.stride, a.E),
                                                                                         rows_of_lanes<decltype(ty), decltype(v)::value>(a.d_logits, a.d_stride, a.E));
            return hipGetLastError();
        });
    });
}

size_t route_plan_bytes(int64_t slots, int E)
{
    if (slots <= BLOCK_SLOTS) return 0;
    const int64_t chunk = plan_chunk(slots);
    return (size_t)((slots + chunk - 1) / chunk) * E * sizeof(int);
}

hipError_t launch_route_plan(const int32_t *ids, const asgd_route_order &o, void *work, hipStream_t s)
{
    const int64_t slots = o.T * o.k, chunk = slots ? plan_chunk(slots) : BLOCK_SLOTS;
    const int chunks = slots ? (int)((slots + chunk - 1) / chunk) : 1;
    int bits = 0;
    while (o.E >> bits) bits++;                       // (E itself stands for none)
    if (chunks > 1) {
        plan_count_kernel<<<chunks, 1024, 0, s>>>(ids, slots, chunk, o.E, bits, (int *)work);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    plan_place_kernel<<<chunks, 1024, (size_t)16 * (o.E + 1) * sizeof(unsigned short), s>>>(ids, o, chunk, chunks, bits, (const int *)work);
    return hipGetLastError();
}

}  // namespace asgd
