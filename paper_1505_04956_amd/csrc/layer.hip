// A whole layer of experts for few rows: what the routing chose, through both matrices of every expert that some row goes to.  An expert's weights are
// read once for all rows: up to sixteen rows are the columns of one matrix instruction, and the columns of rows that do not go to an expert are not used.
//
// The first kernel forms h = f(gate) * up in 32 bits for every slot (a row and one of its choices), the second sums the rows' experts.
#include "four_bits.h"

namespace asgd {

namespace {

constexpr int UP_WAVES = 8, DOWN_WAVES = 16;
constexpr int MOST_SLOTS = ASGD_PRODUCT_RAW_ROWS * ASGD_ROUTE_MAX_CHOSEN;

// ---- which experts have rows --------------------------------------------------------------------------------------
// A bit for each expert that a slot goes to, in the LDS.
__device__ __forceinline__ void mark_experts(const int32_t *ids, int slots, int E, uint32_t *bits)
{
    for (int i = threadIdx.x; i < ASGD_ROUTE_MAX_EXPERTS / 32; i += blockDim.x) bits[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < slots; i += blockDim.x) {
        const int e = ids[i];
        if ((unsigned)e < (unsigned)E) atomicOr(&bits[e >> 5], 1u << (e & 31));
    }
    __syncthreads();
}

// The n-th of them, -1 if there are not so many.  All lanes of a wave.
__device__ __forceinline__ int nth_expert(const uint32_t *bits, int n)
{
    const int lane = threadIdx.x & 63;
    const uint32_t word = lane < ASGD_ROUTE_MAX_EXPERTS / 32 ? bits[lane] : 0;
    const int sum = wave_scan(__popc(word)), before = sum - __popc(word);
    const unsigned long long past = __ballot(sum > n);
    if (!past) return -1;
    const int at = __ffsll((long long)past) - 1;
    uint32_t rest = (uint32_t)__builtin_amdgcn_readlane((int)word, at);
    for (int skip = n - __builtin_amdgcn_readlane(before, at); skip > 0; skip--) rest &= rest - 1;
    return at * 32 + __ffs((int)rest) - 1;
}

// ---- sixteen rows of an expert's weights ----------------------------------------------------------------------------
// A step is a block of 128 columns (8 bits) or a run of 256 (4 bits).  Which rows: a lane's own (row), the first of the sixteen (tile).
template <int BITS> struct Weights;

template <> struct Weights<8> {
    static constexpr int STEP = BLOCK8;
    template <class In> struct Rows {                              // the columns' rows of a step
        RawBlock<In> raw;
        Operand<true> a;
        float scale;
        __device__ __forceinline__ void load(const typename In::T *row, bool there, bool wide, int64_t step, int quarter, int64_t cols)
        {
            raw.load(row, there, wide, step * BLOCK8 + quarter * 32, cols);
        }
        __device__ __forceinline__ void set(bool there)
        {
            v4i lo, hi;
            raw.set(there, scale, lo, hi);
            a.set(lo, hi);
        }
    };
    v4i lo, hi;
    float scale[2];                                                // of the square that the first of the sixteen rows lies in, and of that of the last
    __device__ __forceinline__ void load(const asgd_blocks &w, int64_t steps, int64_t matrix, int64_t row, int64_t tile, int64_t step, int quarter)
    {
        const uint8_t *p = (const uint8_t *)w.values + ((matrix * w.rows + row) * steps + step) * BLOCK8 + quarter * 32;
        lo = *(const v4i *)p;
        hi = *(const v4i *)(p + 16);
        const float *s = w.scales + matrix * blocks8(w.rows) * steps + step;
        scale[0] = s[tile / BLOCK8 * steps];
        scale[1] = s[min(tile + 15, w.rows - 1) / BLOCK8 * steps];
    }
    // the products are added to `sum`, a row of the result for each lane and i
    template <class In> __device__ __forceinline__ v4f times(const Rows<In> &r, int64_t tile, int quarter, v4f sum) const
    {
        Operand<true> b;
        b.set(lo, hi);
        const v4f part = block_product(b, r.a);
        const int second = BLOCK8 - (int)(tile % BLOCK8) - quarter * 4;      // from this i on the lane's rows lie in the second square
#pragma unroll
        for (int i = 0; i < 4; i++) sum[i] = fmaf(part[i], r.scale * (i < second ? scale[0] : scale[1]), sum[i]);
        return sum;
    }
};

template <> struct Weights<4> {
    static constexpr int STEP = RUN4;
    template <class In> struct Rows {
        RawFour<In> raw[2];
        v4i a[2];
        uint32_t scale[2];
        __device__ __forceinline__ void load(const typename In::T *row, bool there, bool wide, int64_t step, int quarter, int64_t cols)
        {
#pragma unroll
            for (int half = 0; half < 2; half++) raw[half].load(row, there, wide, step * RUN4 + half * 128 + quarter * 32, cols);
        }
        __device__ __forceinline__ void set(bool there)
        {
#pragma unroll
            for (int half = 0; half < 2; half++) raw[half].set(there, scale[half], a[half]);
        }
    };
    v4i v[2];
    uint32_t scale[2];
    __device__ __forceinline__ void load(const asgd_blocks &w, int64_t steps, int64_t matrix, int64_t row, int64_t, int64_t step, int quarter)
    {
        const int64_t at = (matrix * w.rows + row) * steps + step;
        const uint8_t *p = (const uint8_t *)w.values + at * RUN4_BYTES + quarter * 16, *s = (const uint8_t *)w.scales + at * RUN4_SCALES + quarter;
#pragma unroll
        for (int half = 0; half < 2; half++) {
            v[half] = *(const v4i *)(p + half * 64);
            scale[half] = s[half * 4];
        }
    }
    template <class In> __device__ __forceinline__ v4f times(const Rows<In> &r, int64_t, int, v4f sum) const
    {
#pragma unroll
        for (int half = 0; half < 2; half++) sum = four_product(v[half], scale[half], r.a[half], r.scale[half], sum);
        return sum;
    }
};

// ---- kernels --------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float activated(float gate, float up, int activation)
{
    const float f = activation == ASGD_ACTIVATION_SILU ? gate / (1.0f + expf(-gate)) : 0.5f * gate * (1.0f + erff(gate * 0.70710678f));
    return f * up;
}

__host__ __device__ inline int64_t h_pitch(int64_t H) { return (H + 3) & ~(int64_t)3; }

// grid: strips of sixteen of H, experts
template <class In, int BITS> __global__ __launch_bounds__(64 * UP_WAVES) void layer_up_kernel(LayerArgs a, bool wide)
{
    typedef Weights<BITS> W;
    __shared__ uint32_t bits[ASGD_ROUTE_MAX_EXPERTS / 32];
    __shared__ v4f parts[UP_WAVES][2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tok = lane & 15, quarter = lane >> 4;
    mark_experts(a.ids, a.T * a.k, a.E, bits);
    const int e = nth_expert(bits, blockIdx.y);
    if (e < 0) return;
    int slot = -1;
    if (tok < a.T)
        for (int j = quarter; j < a.k; j += 4)
            if (a.ids[tok * a.k + j] == e) slot = tok * a.k + j;
    slot = max(slot, __shfl_xor(slot, 16));
    slot = max(slot, __shfl_xor(slot, 32));
    const bool there = slot >= 0;
    const int64_t strip = (int64_t)blockIdx.x * 16, steps = (a.D + W::STEP - 1) / W::STEP, of_lane = min(strip + tok, a.H - 1);
    const typename In::T *row = (const typename In::T *)a.x + (there ? tok : 0) * a.x_stride;
    v4f sum[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    for (int64_t step = wave; step < steps; step += UP_WAVES) {
        W w[2];
        typename W::template Rows<In> r;
#pragma unroll
        for (int n = 0; n < 2; n++) w[n].load(a.up, steps, e, n * a.H + of_lane, n * a.H + strip, step, quarter);
        r.load(row, there, wide, step, quarter, a.D);
        r.set(there);
#pragma unroll
        for (int n = 0; n < 2; n++) sum[n] = w[n].template times<In>(r, n * a.H + strip, quarter, sum[n]);
    }
#pragma unroll
    for (int n = 0; n < 2; n++) parts[wave][n][lane] = sum[n];
    __syncthreads();
    if (wave > 0 || !there) return;
    v4f total[2] = {parts[0][0][lane], parts[0][1][lane]};
#pragma unroll
    for (int w = 1; w < UP_WAVES; w++)
#pragma unroll
        for (int n = 0; n < 2; n++) total[n] += parts[w][n][lane];
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (strip + quarter * 4 + i < a.H) a.h[slot * h_pitch(a.H) + strip + quarter * 4 + i] = activated(total[0][i], total[1][i], a.activation);
}

// grid: strips of sixteen of N.  The waves share the steps of all experts.
template <int BITS, class Out> __global__ __launch_bounds__(64 * DOWN_WAVES) void layer_down_kernel(LayerArgs a, bool wide)
{
    typedef Weights<BITS> W;
    extern __shared__ int16_t slots[];                            // [experts that have rows][sixteen rows]: the slot, -1 without one
    __shared__ uint32_t bits[ASGD_ROUTE_MAX_EXPERTS / 32];
    __shared__ int before[ASGD_ROUTE_MAX_EXPERTS / 32 + 1];       // experts with rows in the words before
    __shared__ int16_t experts[MOST_SLOTS];
    __shared__ v4f parts[DOWN_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tok = lane & 15, quarter = lane >> 4;
    const int all = a.T * a.k;
    mark_experts(a.ids, all, a.E, bits);
    if (wave == 0) {
        const int c = lane < ASGD_ROUTE_MAX_EXPERTS / 32 ? __popc(bits[lane]) : 0, sum = wave_scan(c);
        if (lane <= ASGD_ROUTE_MAX_EXPERTS / 32) before[lane] = sum - c;
    }
    __syncthreads();
    const int met = before[ASGD_ROUTE_MAX_EXPERTS / 32];
    for (int i = threadIdx.x; i < met * 16; i += blockDim.x) slots[i] = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += blockDim.x) {
        const int e = a.ids[i];
        if ((unsigned)e < (unsigned)a.E) {
            const int n = before[e >> 5] + __popc(bits[e >> 5] & ((1u << (e & 31)) - 1));
            slots[n * 16 + i / a.k] = (int16_t)i;
            experts[n] = (int16_t)e;                               // (every slot of an expert: the same number)
        }
    }
    __syncthreads();
    const int64_t strip = (int64_t)blockIdx.x * 16, of_lane = min(strip + tok, a.N - 1);
    const int steps = (int)((a.H + W::STEP - 1) / W::STEP);
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int item = wave; item < met * steps; item += DOWN_WAVES) {
        const int n = item / steps, step = item - n * steps, slot = slots[n * 16 + tok];
        const bool there = slot >= 0;
        W w;
        typename W::template Rows<F32> r;
        w.load(a.down, steps, experts[n], of_lane, strip, step, quarter);
        r.load(a.h + (there ? slot : 0) * h_pitch(a.H), there, wide, step, quarter, a.H);
        const float weight = there ? a.weights[slot] : 0.0f;
        r.set(there);
        const v4f part = w.template times<F32>(r, strip, quarter, v4f{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
        for (int i = 0; i < 4; i++) sum[i] = there ? fmaf(part[i], weight, sum[i]) : sum[i];     // (a scale that is not a number spoils its own expert's rows alone)
    }
    parts[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || tok >= a.T) return;
#pragma unroll
    for (int w = 1; w < DOWN_WAVES; w++) sum += parts[w][lane];
    const int64_t c = strip + quarter * 4;
    store_four<Out>((typename Out::T *)a.out + tok * a.out_stride + c, a.N - c, a.wide_out, sum);
}

// The experts of few rows in 4 bits in one launch, without an order: a workgroup takes sixteen rows of the weights of every expert of one row of x
// (blockIdx.y), which it brings to 4 bits itself.
template <class In, class Out> __global__ __launch_bounds__(64 * DOWN_WAVES) void direct_four_kernel(LayerArgs a, bool wide)
{
    typedef Weights<4> W;
    __shared__ v4f parts[DOWN_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tok = lane & 15, quarter = lane >> 4;
    const int64_t t = blockIdx.y, strip = (int64_t)blockIdx.x * 16, of_lane = min(strip + tok, a.N - 1);
    const int steps = (int)runs4(a.H);
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int step = wave; step < steps; step += DOWN_WAVES) {
        typename W::template Rows<In> r;
        r.load((const typename In::T *)a.x + t * a.x_stride, tok == 0, wide, step, quarter, a.H);
        r.set(tok == 0);
        for (int j = 0; j < a.k; j++) {
            const int e = a.ids[t * a.k + j];
            if ((unsigned)e >= (unsigned)a.E) continue;            // (all lanes or none)
            W w;
            w.load(a.down, steps, e, of_lane, strip, step, quarter);
            const v4f part = w.template times<In>(r, strip, quarter, v4f{0.0f, 0.0f, 0.0f, 0.0f});
            const float weight = a.weights[t * a.k + j];
#pragma unroll
            for (int i = 0; i < 4; i++) sum[i] = fmaf(part[i], weight, sum[i]);
        }
    }
    parts[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || tok > 0) return;
#pragma unroll
    for (int w = 1; w < DOWN_WAVES; w++) sum += parts[w][lane];
    const int64_t c = strip + quarter * 4;
    store_four<Out>((typename Out::T *)a.out + t * a.out_stride + c, a.N - c, a.wide_out, sum);
}

bool rows_wide(const void *p, int64_t stride, int type) { return (uintptr_t)p % 16 == 0 && stride * (int64_t)type_size(type) % 16 == 0; }
unsigned strips_of(int64_t n) { return (unsigned)((n + 15) / 16); }

}  // namespace

size_t layer_bytes(int64_t T, int k, int64_t H) { return sizeof(float) * (size_t)(T * k) * (size_t)h_pitch(H); }

hipError_t launch_layer(const LayerArgs &a, int x_type, int type, hipStream_t s)
{
    const int most = a.T * a.k < a.E ? a.T * a.k : a.E;
    const bool four = a.up.form == ASGD_BLOCKS_FOURS;
    const dim3 grid(strips_of(a.H), (unsigned)most);
    const hipError_t e = with_type(x_type, [&](auto in) {
        typedef decltype(in) In;
        if (four) layer_up_kernel<In, 4><<<grid, 64 * UP_WAVES, 0, s>>>(a, rows_wide(a.x, a.x_stride, x_type));
        else layer_up_kernel<In, 8><<<grid, 64 * UP_WAVES, 0, s>>>(a, rows_wide(a.x, a.x_stride, x_type));
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    return with_type(type, [&](auto out) {
        typedef decltype(out) Out;
        const size_t lds = (size_t)most * 16 * sizeof(int16_t);
        if (four) layer_down_kernel<4, Out><<<strips_of(a.N), 64 * DOWN_WAVES, lds, s>>>(a, true);
        else layer_down_kernel<8, Out><<<strips_of(a.N), 64 * DOWN_WAVES, lds, s>>>(a, true);
        return hipGetLastError();
    });
}

hipError_t launch_direct_four(const LayerArgs &a, int x_type, int type, hipStream_t s)
{
    const dim3 grid(strips_of(a.N), (unsigned)a.T);
    return with_type(x_type, [&](auto in) {
        return with_type(type, [&](auto out) {
            direct_four_kernel<decltype(in), decltype(out)><<<grid, 64 * DOWN_WAVES, 0, s>>>(a, rows_wide(a.x, a.x_stride, x_type));
            return hipGetLastError();
        });
    });
}

}  // namespace asgd
