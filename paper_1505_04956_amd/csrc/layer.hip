// A whole layer of experts for few rows in three launches, or two.  An expert's weights are read once for all rows: up to sixteen rows are the columns of one
// matrix instruction, and the columns of rows that do not go to an expert are not used.
//
//   choose  one workgroup routes the rows and lists the experts that have any; the others bring a row of x each to 8 or 4 bits (or, for very few rows, every
//           workgroup of the next part does both)
//   up      a workgroup forms h = f(gate) * up, 32-bit, of sixteen of an expert's hidden columns for all of its rows
//   down    a workgroup sums sixteen columns of the result over all experts; its waves share the experts' blocks
//
// The weights' way from memory bounds the second and third: sixteen rows of eight of 128 experts of 4096 x 1024 in 4 bits 67 us (5.4 TB/s) and 38 (4.7), one row of six of 64
// of 2048 x 1408 in 8 bits, 34.6 and 17.3 MB, 11.9 us and 8.0, where a chain of loads (lists, rows, weights) is as long as what they bring (those weights lay in the last cache; from memory both
// take 1.5 us more); choose 3.5 to 6 us, a launch and a row's routing.
#include "four_bits.h"
#include "route_row.h"

namespace asgd {

namespace {

constexpr int UP_WAVES = 4, DOWN_WAVES = 16, COLUMNS = 16;
// Up to so many rows, experts, steps of all rows, and workgroups times rows (which all route and bring to 8 or 4 bits the same) one launch does the first two
// parts.  Layers in 8 bits so and else, us of a run of them in a graph: one row of six of 64 experts of 2048 x 1408 (528 workgroups times rows) 20.6 and 22.8, two rows (2112) 26.2 and
// 28.5, two of eight (2816) 34.4 and 34.9, three of four (3168) 31.9 and 28.3, four of six (8448) 45.9 and 40.8; three of eight of 64 of 1024 x 704 (3168) 21.6 and 23.0; five of four
// of 40 of 512 x 512 (3200) 15.7 and 14.8; six of three of 64 (3456) 16.0 and 14.7; in 4 bits five of five of 100 of 1000 x 700 (5500) 22.5 and 20.4.
constexpr int FEW_ROWS = 8, FEW_EXPERTS = 256, FEW_STEPS = 128, FEW_GROUPS = 2560;
constexpr int MOST_SLOTS = ASGD_PRODUCT_RAW_ROWS * ASGD_ROUTE_MAX_CHOSEN, WORDS = ASGD_ROUTE_MAX_EXPERTS / 32;
static_assert(ASGD_PRODUCT_RAW_ROWS == COLUMNS, "");

// A step of a contraction is what a row has in 128 bytes: a block of 128 columns in 8 bits, a run of 256 in 4.
constexpr int STEP_BYTES = 128;
__host__ __device__ inline int64_t steps_of(int bits, int64_t cols) { return bits == 8 ? blocks8(cols) : runs4(cols); }

// Scratch of a call, each part at a multiple of sixteen bytes.
struct Scratch {
    int32_t *met, *experts;       // experts that have rows: how many, which, in ascending order
    int16_t *slots;               // [met][sixteen rows]: the slot t * k + j with which row t goes to it, -1 if it does not
    uint8_t *x, *x_scales;        // rows of x in 8 bits, a float for each step, or in 4, eight bytes for each
    float *h;                     // [T * k] rows, h_pitch() apart
};
__host__ __device__ inline int64_t h_pitch(int64_t H) { return (H + 3) & ~(int64_t)3; }

size_t scratch_of(int64_t T, int k, int64_t E, int64_t D, int64_t H, char *at, Scratch &s)
{
    const int64_t most = T * k < E ? T * k : E, steps = blocks8(D);        // (enough for either)
    size_t n = 0;
    const auto take = [&](size_t bytes) { char *p = at + n; n += (bytes + 15) & ~(size_t)15; return p; };
    s.met = (int32_t *)take(4);
    s.experts = (int32_t *)take(4 * most);
    s.slots = (int16_t *)take(2 * COLUMNS * most);
    s.x = (uint8_t *)take(T * steps * STEP_BYTES);
    s.x_scales = (uint8_t *)take(T * steps * 8);
    s.h = (float *)take(sizeof(float) * T * k * h_pitch(H));
    return n;
}

// ---- bringing rows to 8 or 4 bits -----------------------------------------------------------------------------------
// (by `threads` threads, of which this is number `me`)
template <int BITS, class T> __device__ __forceinline__ void bring_row(const T *row, int64_t cols, uint8_t *values, uint8_t *scales, int me, int threads)
{
    typedef Parts<BITS> P;
    const int part = me % P::LANES;
    const int64_t steps = steps_of(BITS, cols);
    for (int64_t step = me / P::LANES; step < steps; step += threads / P::LANES) {
        float v[8];
        eight_of(row, (step * P::LANES + part) * 8, cols, v);
        typename P::Scale scale;
        *(typename P::Bytes *)(values + step * STEP_BYTES + part * P::BYTES) = P::to(v, scale);
        P::put_scale(scales + step * P::SCALES, part, scale);
    }
}

// ---- sixteen rows of an expert's weights, and the columns that they are multiplied by ------------------------------------
template <int BITS> struct Weights;                               // of a step.  row: the lane's operand's, first: the first of the four rows of the result that it gets
template <int BITS> struct Columns;                               // of a step, a lane's 32 or two times 32 of row lane % 16

template <> struct Columns<8> {
    v4i lo, hi;
    float scale;
    __device__ __forceinline__ void load(const uint8_t *values, const uint8_t *scales, int quarter)
    {
        lo = *(const v4i *)(values + quarter * 32);
        hi = *(const v4i *)(values + quarter * 32 + 16);
        scale = *(const float *)scales;
    }
};
template <> struct Weights<8> {
    v4i lo, hi;
    float scale[2];                                                // of the square that the first of the lane's four rows lies in, and of that of the last (a load of the lane's
                                                                   // own: the same for all, it would be a scalar one, which the compiler puts after the wait for the values)
    __device__ __forceinline__ void load(const asgd_blocks &w, int64_t steps, int64_t matrix, int64_t row, int64_t first, int64_t step, int quarter)
    {
        const uint8_t *p = (const uint8_t *)w.values + ((matrix * w.rows + row) * steps + step) * BLOCK8 + quarter * 32;
        lo = *(const v4i *)p;
        hi = *(const v4i *)(p + 16);
        const float *s = w.scales + matrix * blocks8(w.rows) * steps + step;
        scale[0] = s[min(first, w.rows - 1) / BLOCK8 * steps];
        scale[1] = s[min(first + 3, w.rows - 1) / BLOCK8 * steps];
    }
    // adds the products times `factor` to `sum`, a row of the result for each lane and i
    __device__ __forceinline__ v4f times(const Columns<8> &c, int64_t first, float factor, v4f sum) const
    {
        Operand<true> a, b;
        a.set(c.lo, c.hi);
        b.set(lo, hi);
        const v4f part = block_product(b, a);
        const int second = BLOCK8 - (int)(first % BLOCK8);         // from this i on they lie in the second
#pragma unroll
        for (int i = 0; i < 4; i++) sum[i] = fmaf(part[i], c.scale * factor * (i < second ? scale[0] : scale[1]), sum[i]);
        return sum;
    }
};

template <> struct Columns<4> {
    v4i v[2];
    uint2 scales;
    __device__ __forceinline__ void load(const uint8_t *values, const uint8_t *of, int quarter)
    {
#pragma unroll
        for (int half = 0; half < 2; half++) v[half] = *(const v4i *)(values + half * 64 + quarter * 16);
        scales = *(const uint2 *)of;
    }
};
template <> struct Weights<4> {
    v4i v[2];
    uint2 scales;                                                  // all eight of a run: two loads of a byte each cost as much as the values' do
    __device__ __forceinline__ void load(const asgd_blocks &w, int64_t steps, int64_t matrix, int64_t row, int64_t, int64_t step, int quarter)
    {
        const int64_t at = (matrix * w.rows + row) * steps + step;
        const uint8_t *p = (const uint8_t *)w.values + at * RUN4_BYTES + quarter * 16;
#pragma unroll
        for (int half = 0; half < 2; half++) v[half] = *(const v4i *)(p + half * 64);
        scales = *(const uint2 *)((const uint8_t *)w.scales + at * RUN4_SCALES);
    }
    __device__ __forceinline__ v4f times(const Columns<4> &c, v4f sum) const
    {
        const int at = (threadIdx.x >> 4 & 3) * 8;                 // the lane's quarter
        sum = four_product(v[0], scales.x >> at & 255, c.v[0], c.scales.x >> at & 255, sum);
        return four_product(v[1], scales.y >> at & 255, c.v[1], c.scales.y >> at & 255, sum);
    }
    __device__ __forceinline__ v4f times(const Columns<4> &c, int64_t, float factor, v4f sum) const
    {
        const v4f part = times(c, v4f{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
        for (int i = 0; i < 4; i++) sum[i] = fmaf(part[i], factor, sum[i]);
        return sum;
    }
};

// ---- up -----------------------------------------------------------------------------------------------------------------
// (1 + erf(v) is formed as erfc(-v): far below zero the sum would cancel, and from a gate of -5.6 on be zero, so that blocks of such h would be lost.  0.1 us of 112: sixteen rows of eight of 128 experts)
__device__ __forceinline__ float activated(float gate, float up, int activation)
{
    const float f = activation == ASGD_ACTIVATION_SILU ? gate / (1.0f + expf(-gate)) : 0.5f * gate * erfcf(gate * -0.70710678f);
    return f * up;
}

// Sixteen rows of the gate and the sixteen that they multiply; a workgroup's waves share the steps, and the loads of AHEAD of a wave's steps are on their way together.
// slot: of the lane's column; x, x_scales: of that column's row.
template <int BITS> __device__ __forceinline__ void form_h(const LayerArgs &a, const Scratch &s, v4f (*parts)[2][64], int e, int slot, const uint8_t *x, const uint8_t *x_scales)
{
    constexpr int AHEAD = 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tok = lane & 15, quarter = lane >> 4;
    const int64_t strip = (int64_t)blockIdx.x * 16;
    const int steps = (int)steps_of(BITS, a.D);
    const int64_t first[2] = {strip + quarter * 4, a.H + strip + quarter * 4}, of_lane = min(strip + tok, a.H - 1);
    v4f sum[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    for (int step0 = wave; step0 < steps; step0 += UP_WAVES * AHEAD) {
        Weights<BITS> w[AHEAD][2];
        Columns<BITS> c[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
            const int step = step0 + i * UP_WAVES;
            if (step >= steps) break;
#pragma unroll
            for (int m = 0; m < 2; m++) w[i][m].load(a.up, steps, e, m * a.H + of_lane, first[m], step, quarter);
            c[i].load(x + (int64_t)step * STEP_BYTES, x_scales + (int64_t)step * Parts<BITS>::SCALES, quarter);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
            if (step0 + i * UP_WAVES >= steps) break;
#pragma unroll
            for (int m = 0; m < 2; m++) {
                if constexpr (BITS == 8) sum[m] = w[i][m].times(c[i], first[m], 1.0f, sum[m]);
                else sum[m] = w[i][m].times(c[i], sum[m]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < 2; m++) parts[wave][m][lane] = sum[m];
    __syncthreads();
    if (wave > 0 || slot < 0) return;
    v4f gate = parts[0][0][lane], up = parts[0][1][lane];
#pragma unroll
    for (int w = 1; w < UP_WAVES; w++) {
        gate += parts[w][0][lane];
        up += parts[w][1][lane];
    }
    const int64_t c = strip + quarter * 4;
    if (c >= a.H) return;
    v4f h;
#pragma unroll
    for (int i = 0; i < 4; i++) h[i] = c + i < a.H ? activated(gate[i], up[i], a.activation) : 0.0f;
    *(v4f *)(s.h + slot * h_pitch(a.H) + c) = h;                   // (a row has a multiple of four)
}

// ---- which experts have rows ------------------------------------------------------------------------------------------------
// In the LDS: what a workgroup knows of the routing.
template <int SLOTS> struct Chosen {
    int32_t ids[SLOTS];
    float weights[SLOTS];
    uint32_t bits[WORDS];                                          // of each expert whether it has rows
    int before[WORDS + 1];                                         // experts with rows in the words before
    int16_t experts[SLOTS];
};

// Routes the rows, a wave each, and marks their experts.  The whole workgroup.
template <class Ty, int V, int SLOTS> __device__ __forceinline__ void choose(RouteArgs r, const LayerArgs &a, Chosen<SLOTS> &c, bool wide)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    for (int i = threadIdx.x; i < WORDS; i += blockDim.x) c.bits[i] = 0;
    r.ids = c.ids;
    r.weights = c.weights;
#pragma unroll 1
    for (int t = wave; t < a.T; t += waves) {
        float bias[V];
        load_bias<V>(r.bias, r.E, lane, bias);
        const Lane<Ty, V> row = load_lane<Ty, V>((const typename Ty::T *)r.logits + t * r.stride, lane * V, r.E, wide);
        route_row<Ty, V, true>(r, t, lane, row, bias);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * a.k; i += blockDim.x) {
        const int e = c.ids[i];
        if (e >= 0) atomicOr(&c.bits[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
}

// Writes ids, weights and the scratch's lists.  The whole workgroup.
template <int SLOTS> __device__ __forceinline__ void list_chosen(const LayerArgs &a, const Scratch &s, Chosen<SLOTS> &c)
{
    const int lane = threadIdx.x & 63, all = a.T * a.k;
    if (threadIdx.x < 64) {
        const int n = lane < WORDS ? __popc(c.bits[lane]) : 0, sum = wave_scan(n);
        if (lane <= WORDS) c.before[lane] = sum - n;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += blockDim.x) {
        const int e = c.ids[i];
        a.ids[i] = e;
        a.weights[i] = c.weights[i];
        if (e >= 0) c.experts[c.before[e >> 5] + __popc(c.bits[e >> 5] & ((1u << (e & 31)) - 1))] = (int16_t)e;      // (every slot of an expert: the same number)
    }
    __syncthreads();
    const int met = c.before[WORDS];
    if (threadIdx.x == 0) *s.met = met;
    for (int i = threadIdx.x; i < met; i += blockDim.x) s.experts[i] = c.experts[i];
    for (int i = threadIdx.x; i < met * COLUMNS; i += blockDim.x) {
        const int e = c.experts[i / COLUMNS], t = i % COLUMNS;
        int slot = -1;
        for (int j = 0; t < a.T && j < a.k; j++)
            if (c.ids[t * a.k + j] == e) slot = t * a.k + j;
        s.slots[i] = (int16_t)slot;
    }
}

template <int BITS> __device__ __forceinline__ void bring_x(const LayerArgs &a, int t, uint8_t *values, uint8_t *scales, int me, int threads)
{
    const int64_t at = t * a.x_stride;
    if (a.x_type == ASGD_TYPE_F32) bring_row<BITS>((const float *)a.x + at, a.D, values, scales, me, threads);
    else if (a.x_type == ASGD_TYPE_BF16) bring_row<BITS>((const __bf16 *)a.x + at, a.D, values, scales, me, threads);
    else bring_row<BITS>((const _Float16 *)a.x + at, a.D, values, scales, me, threads);
}

// ---- many workgroups: choose, then up -------------------------------------------------------------------------------------------
// a wave for each row, but for the most experts, which take the registers of two
template <int V> constexpr int CHOOSE_THREADS = V < 16 ? 1024 : 512;
template <class Ty, int V> __global__ __launch_bounds__(CHOOSE_THREADS<V>) void layer_choose_kernel(RouteArgs r, LayerArgs a, Scratch s, bool wide)
{
    __shared__ Chosen<MOST_SLOTS> chosen;
    if (blockIdx.x > 0) {
        const int t = blockIdx.x - 1;
        if (a.up.form == ASGD_BLOCKS_FOURS) bring_x<4>(a, t, s.x + t * runs4(a.D) * STEP_BYTES, s.x_scales + t * runs4(a.D) * Parts<4>::SCALES, threadIdx.x, blockDim.x);
        else bring_x<8>(a, t, s.x + t * blocks8(a.D) * STEP_BYTES, s.x_scales + t * blocks8(a.D) * Parts<8>::SCALES, threadIdx.x, blockDim.x);
        return;
    }
    choose<Ty, V>(r, a, chosen, wide);
    list_chosen(a, s, chosen);
}

// grid: strips of sixteen of H, experts.  (Small workgroups spread evenly: with 32 of H and eight waves one token's took 14.1 us for 12.)
template <int BITS> __global__ __launch_bounds__(64 * UP_WAVES, 4) void layer_up_kernel(LayerArgs a, Scratch s)
{
    __shared__ v4f parts[UP_WAVES][2][64];
    const int n = blockIdx.y, met = *s.met, e = s.experts[n], slot = s.slots[n * COLUMNS + (threadIdx.x & 15)];
    if (n >= met) return;
    const int64_t row = slot < 0 ? 0 : threadIdx.x & 15, steps = steps_of(BITS, a.D);
    form_h<BITS>(a, s, parts, e, slot, s.x + row * steps * STEP_BYTES, s.x_scales + row * steps * Parts<BITS>::SCALES);
}

// ---- few workgroups: both in one launch -------------------------------------------------------------------------------------------
// Every workgroup routes the rows and brings them to 8 or 4 bits for itself; the first writes the lists that the next launch reads.
template <class Ty, int V, int BITS> __global__ __launch_bounds__(64 * UP_WAVES, 4) void layer_choose_up_kernel(RouteArgs r, LayerArgs a, Scratch s, bool wide)
{
    __shared__ Chosen<FEW_ROWS * ASGD_ROUTE_MAX_CHOSEN> chosen;
    __shared__ v4f parts[UP_WAVES][2][64];
    __shared__ __align__(16) uint8_t x[FEW_STEPS * STEP_BYTES], x_scales[FEW_STEPS * 8];
    const int lane = threadIdx.x & 63, tok = lane & 15, steps = (int)steps_of(BITS, a.D);
    // (where there are fewer rows than waves, by those that have none to route)
    const int routing = a.T < UP_WAVES ? 64 * a.T : 0;
    if ((int)threadIdx.x >= routing)
        for (int t = 0; t < a.T; t++) bring_x<BITS>(a, t, x + t * steps * STEP_BYTES, x_scales + t * steps * Parts<BITS>::SCALES, threadIdx.x - routing, blockDim.x - routing);
    choose<Ty, V>(r, a, chosen, wide);
    if (blockIdx.x == 0 && blockIdx.y == 0) list_chosen(a, s, chosen);
    // the expert of this workgroup: the blockIdx.y-th that has rows
    const uint32_t word = lane < WORDS ? chosen.bits[lane] : 0;
    const int sum = wave_scan(__popc(word)), n = blockIdx.y;
    const unsigned long long past = __ballot(sum > n);
    if (!past) return;                                             // (all waves alike)
    const int at = __ffsll((long long)past) - 1;
    uint32_t rest = (uint32_t)__builtin_amdgcn_readlane((int)word, at);
    for (int skip = n - __builtin_amdgcn_readlane(sum - __popc(word), at); skip > 0; skip--) rest &= rest - 1;
    const int e = at * 32 + __ffs((int)rest) - 1;
    int slot = -1;
    for (int j = lane >> 4; tok < a.T && j < a.k; j += 4)
        if (chosen.ids[tok * a.k + j] == e) slot = tok * a.k + j;
    slot = max(slot, __shfl_xor(slot, 16));
    slot = max(slot, __shfl_xor(slot, 32));
    const int row = slot < 0 ? 0 : tok;
    form_h<BITS>(a, s, parts, e, slot, x + row * steps * STEP_BYTES, x_scales + row * steps * Parts<BITS>::SCALES);
}

// ---- down ---------------------------------------------------------------------------------------------------------------
// An item is G neighbouring steps of an expert; the waves of a workgroup take items in turn.  A wave brings the item's part of h to 8 or 4 bits itself, sixteen or 32
// lanes a row and step, and hands it round through the LDS; the weights of its next items are on their way meanwhile.
//
// G = 2, for up to eight rows: the sixteen rows of the matrix instruction are eight of the weights with two steps each, and its columns eight rows of h with
// the same two; what belongs together is half of what it gives.  So a workgroup takes eight columns of the result, and there are twice as many of them.
template <int BITS, int G, class Out> __global__ __launch_bounds__(64 * DOWN_WAVES, 4) void layer_down_kernel(LayerArgs a, Scratch s, int most)
{
    typedef Parts<BITS> P;
    constexpr int PITCH = STEP_BYTES + 16, GROUPS = 64 / P::LANES, AHEAD = 2, R = COLUMNS / G;
    __shared__ int16_t slots[MOST_SLOTS * COLUMNS];
    __shared__ int16_t experts[MOST_SLOTS];
    __shared__ float weights[MOST_SLOTS];
    __shared__ __align__(16) uint8_t columns[DOWN_WAVES][COLUMNS * PITCH];
    __shared__ __align__(16) uint8_t scales[DOWN_WAVES][COLUMNS * 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tok = lane & 15, quarter = lane >> 4;
    const int row = tok % R, g = tok / R;                          // of the weights and of x; which of the item's steps
    // (all that there can be: how many there are is on its way as well)
    for (int i = threadIdx.x; i < most * COLUMNS; i += blockDim.x) slots[i] = s.slots[i];
    for (int i = threadIdx.x; i < most; i += blockDim.x) experts[i] = (int16_t)s.experts[i];
    for (int i = threadIdx.x; i < a.T * a.k; i += blockDim.x) weights[i] = a.weights[i];
    const int met = *s.met, steps = (int)steps_of(BITS, a.H), each = (steps + G - 1) / G, items = met * each;
    __syncthreads();
    const int64_t strip = (int64_t)blockIdx.x * R, of_lane = min(strip + row, a.N - 1), first = strip + quarter % (R / 4) * 4;
    const int part = lane % P::LANES, group = lane / P::LANES;

    struct Item {
        Weights<BITS> w;
        float h[8];
        int slot, step;           // of the lane's column (-1: not used); the first of the item
        uint32_t rows;            // rows of x that go to the expert
    };
    const auto nth_row = [](uint32_t rows, int n) {
        for (; n > 0; n--) rows &= rows - 1;
        return __ffs((int)rows) - 1;
    };
    // the at-th used column (the last one if there are fewer), and its part of h
    const auto column_of = [&](uint32_t rows, int at) {
        const int last = min(at, __popc(rows) * G - 1);
        return nth_row(rows, last / G) + last % G * R;
    };
    const auto take_h = [&](int n, int step, int column, float (&h)[8]) {
        eight_of(s.h + slots[n * COLUMNS + column % R] * h_pitch(a.H), ((int64_t)(step + column / R) * P::LANES + part) * 8, a.H, h);
    };
    const auto fetch = [&](int item, Item &i) {
        const int n = item / each;
        i.step = (item - n * each) * G;
        i.slot = slots[n * COLUMNS + row];
        i.rows = (uint32_t)__ballot(i.slot >= 0) & ((1u << R) - 1);
        i.w.load(a.down, steps, experts[n], of_lane, first, min(i.step + g, steps - 1), quarter);
        take_h(n, i.step, column_of(i.rows, group), i.h);
    };
    uint8_t *const mine = columns[wave], *const my_scales = scales[wave];
    const auto put = [&](int column, const float (&h)[8]) {
        typename P::Scale scale;
        *(typename P::Bytes *)(mine + column * PITCH + part * P::BYTES) = P::to(h, scale);
        P::put_scale(my_scales + column * P::SCALES, part, scale);
    };
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    const auto use = [&](int item, const Item &i) {
        const int count = __popc(i.rows) * G;
        put(column_of(i.rows, group), i.h);
        for (int at = GROUPS; at < count; at += GROUPS) {
            float h[8];
            const int column = column_of(i.rows, at + group);
            take_h(item / each, i.step, column, h);
            put(column, h);
        }
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
        Columns<BITS> c;
        c.load(mine + tok * PITCH, my_scales + tok * P::SCALES, quarter);
        // (what a step past the last has of h is zeros)
        const bool there = i.slot >= 0 && (G == 1 || quarter * 4 / R == g);
        const v4f got = i.w.times(c, first, there ? weights[i.slot] : 0.0f, sum);
#pragma unroll
        for (int k = 0; k < 4; k++) sum[k] = there ? got[k] : sum[k];       // (what is not a number in a column that is not used stays there)
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
    };
    Item held[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; i++)
        if (wave + i * DOWN_WAVES < items) fetch(wave + i * DOWN_WAVES, held[i]);
    for (int item = wave; item < items;)
#pragma unroll
        for (int i = 0; i < AHEAD; i++) {
            if (item >= items) break;
            use(item, held[i]);
            if (item + AHEAD * DOWN_WAVES < items) fetch(item + AHEAD * DOWN_WAVES, held[i]);
            item += DOWN_WAVES;
        }
    __syncthreads();
    v4f(*const sums)[64] = (v4f(*)[64])columns;
    static_assert(sizeof(columns) >= DOWN_WAVES * 64 * sizeof(v4f), "");
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || quarter * 4 >= R || tok >= a.T) return;
#pragma unroll
    for (int w = 0; w < DOWN_WAVES; w++)
#pragma unroll
        for (int m = 0; m < G; m++)
            if (w + m > 0) sum += sums[w][lane + m * (R / 4 * 16 + R)];
    const int64_t c = strip + quarter * 4;
    store_four<Out>((typename Out::T *)a.out + tok * a.out_stride + c, min(a.N - c, (int64_t)4), a.wide_out, sum);
}

// ---- experts of one matrix ------------------------------------------------------------------------------------------------
// The experts of few rows in 4 bits in one launch, without an order: a workgroup takes sixteen rows of the weights of every expert of one row of x
// (blockIdx.y), which it brings to 4 bits, CHUNK runs at a time.  Its waves share the runs and, where there are fewer runs than waves, the choices; the weights of EXPERTS of them are on
// their way at a time.
template <class In, class Out, int WAVES> __global__ __launch_bounds__(64 * WAVES) void direct_four_kernel(DirectArgs a)
{
    constexpr int EXPERTS = 4, CHUNK = 32;
    __shared__ v4f parts[WAVES][64];
    __shared__ __align__(16) uint8_t columns[CHUNK * STEP_BYTES], scales[CHUNK * RUN4_SCALES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tok = lane & 15, quarter = lane >> 4;
    const int64_t t = blockIdx.y, strip = (int64_t)blockIdx.x * 16, of_lane = min(strip + tok, a.N - 1);
    const int steps = (int)runs4(a.K), share = steps * 4 <= WAVES ? 4 : steps * 2 <= WAVES ? 2 : 1;       // waves that share a run's choices
    const int32_t *ids = a.ids + t * a.k;
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    Weights<4> w[EXPERTS];
    const auto id_of = [&](int j) { return j < a.k && (unsigned)ids[j] < (unsigned)a.E ? ids[j] : -1; };       // (the same for all lanes)
    const auto fetch = [&](int j0, int step) {
#pragma unroll
        for (int i = 0; i < EXPERTS; i++) {
            const int e = id_of(j0 + i * share);
            if (e >= 0) w[i].load(a.w, steps, e, of_lane, strip, step, quarter);
        }
    };
    const int of_choice = wave % share, first = wave / share, apart = WAVES / share;
    for (int chunk = 0; chunk < steps; chunk += CHUNK) {
        const int end = min(chunk + CHUNK, steps);
        if (chunk + first < end) fetch(of_choice, chunk + first);
        if (chunk > 0) __syncthreads();
        bring_row<4>((const typename In::T *)a.x + t * a.x_stride + (int64_t)chunk * RUN4, min(a.K - (int64_t)chunk * RUN4, (int64_t)CHUNK * RUN4), columns, scales, threadIdx.x, blockDim.x);
        __syncthreads();
        for (int step = chunk + first; step < end; step += apart)
            for (int j0 = of_choice; j0 < a.k; j0 += EXPERTS * share) {
                if (step > chunk + first || j0 > of_choice) fetch(j0, step);
                Columns<4> c;
                c.load(columns + (step - chunk) * STEP_BYTES, scales + (step - chunk) * RUN4_SCALES, quarter);       // (all sixteen columns: the one row)
#pragma unroll
                for (int i = 0; i < EXPERTS; i++)
                    if (id_of(j0 + i * share) >= 0) sum = w[i].times(c, strip, a.weights[t * a.k + j0 + i * share], sum);
            }
    }
    parts[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || tok > 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; w++) sum += parts[w][lane];
    const int64_t c = strip + quarter * 4;
    store_four<Out>((typename Out::T *)a.out + t * a.out_stride + c, a.N - c, a.wide_out, sum);
}

unsigned strips_of(int64_t n, int rows) { return (unsigned)((n + rows - 1) / rows); }

}  // namespace

size_t layer_bytes(int64_t T, int k, int64_t E, int64_t D, int64_t H)
{
    Scratch s;
    return scratch_of(T, k, E, D, H, nullptr, s);
}

hipError_t launch_layer(const LayerArgs &a, const RouteArgs &r, int logits_type, int type, void *work, hipStream_t s)
{
    Scratch w;
    scratch_of(a.T, a.k, a.E, a.D, a.H, (char *)work, w);
    const unsigned most = (unsigned)(a.T * a.k < a.E ? a.T * a.k : a.E);
    const bool four = a.up.form == ASGD_BLOCKS_FOURS;
    const dim3 grid(strips_of(a.H, 16), most);
    const bool together = a.T <= FEW_ROWS && a.E <= FEW_EXPERTS && a.T * steps_of(four ? 4 : 8, a.D) <= FEW_STEPS && (int64_t)grid.x * grid.y * a.T <= FEW_GROUPS;
    hipError_t e = with_type(logits_type, [&](auto ty) {
        return with_width(a.E, [&](auto v) {
            typedef decltype(ty) Ty;
            constexpr int V = decltype(v)::value;
            const bool wide = rows_of_lanes<Ty, V>(r.logits, r.stride, r.E);
            if constexpr (V * 64 <= FEW_EXPERTS)
                if (together) {
                    if (four) layer_choose_up_kernel<Ty, V, 4><<<grid, 64 * UP_WAVES, 0, s>>>(r, a, w, wide);
                    else layer_choose_up_kernel<Ty, V, 8><<<grid, 64 * UP_WAVES, 0, s>>>(r, a, w, wide);
                    return hipGetLastError();
                }
            layer_choose_kernel<Ty, V><<<1 + a.T, CHOOSE_THREADS<V>, 0, s>>>(r, a, w, wide);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess) return e;
    if (!together) {
        if (four) layer_up_kernel<4><<<grid, 64 * UP_WAVES, 0, s>>>(a, w);
        else layer_up_kernel<8><<<grid, 64 * UP_WAVES, 0, s>>>(a, w);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    return with_type(type, [&](auto out) {
        const auto go = [&](auto bits, auto group) {
            constexpr int G = decltype(group)::value;
            layer_down_kernel<decltype(bits)::value, G, decltype(out)><<<strips_of(a.N, COLUMNS / G), 64 * DOWN_WAVES, 0, s>>>(a, w, (int)most);
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> bits4;
        const std::integral_constant<int, 8> bits8;
        if (a.T <= 8) four ? go(bits4, two) : go(bits8, two);
        else four ? go(bits4, one) : go(bits8, one);
        return hipGetLastError();
    });
}

hipError_t launch_direct_four(const DirectArgs &a, int x_type, int type, hipStream_t s)
{
    const dim3 grid(strips_of(a.N, 16), (unsigned)a.T);
    return with_type(x_type, [&](auto in) {
        return with_type(type, [&](auto out) {
            // Sixteen waves where there is a workgroup for each compute unit at most, four where more than one shares it: six experts of 2048 x 2048, 128 workgroups,
            // 7.3 us and 10.0; four rows of four, 512, 10.8 and 10.6; 24 of five of 1000 x 1100, 1656, 23.0 and 15.1; 64 of two of 512 x 512, 2048, 15.7 and 6.4
            if ((int64_t)grid.x * grid.y <= 256) direct_four_kernel<decltype(in), decltype(out), 16><<<grid, 64 * 16, 0, s>>>(a);
            else direct_four_kernel<decltype(in), decltype(out), 4><<<grid, 64 * 4, 0, s>>>(a);
            return hipGetLastError();
        });
    });
}

}  // namespace asgd
