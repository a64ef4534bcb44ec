// The weighted sum of a row's experts, out[t] = sum_j w[t, j] y[place(t, j)], and the gradient of its weights, dw[t, j] = d_out[t] . y[place(t, j)]:
// both read every row of y once, in 32 bits, and memory bounds them.  What is read or written once passes by the second cache: y that the products
// have left in the last one is found there (a training step of 8192 rows of four experts, 1024 x 1024: 455 us; kept, 477).
// 4096 rows of four experts, 2048 columns: 30 us each, 5.1 TB/s.
#include "experts_internal.h"

namespace asgd {

namespace {

constexpr int SPAN = 1024;                 // columns a workgroup of 256 takes, four a thread

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i2 __attribute__((ext_vector_type(2)));

// ONCE: nobody reads it again soon, and it passes by the second cache
template <class Ty, bool ONCE> __device__ __forceinline__ float4 load4(const typename Ty::T *p, int64_t left, bool wide)
{
    typedef typename Ty::T T;
    if (wide && left >= 4) {
        if constexpr (sizeof(T) == 4) {
            const f4 v = ONCE ? __builtin_nontemporal_load((const f4 *)p) : *(const f4 *)p;
            return make_float4(v.x, v.y, v.z, v.w);
        }
        const i2 v = ONCE ? __builtin_nontemporal_load((const i2 *)p) : *(const i2 *)p;
        T u[4];
        *(i2 *)u = v;
        return make_float4((float)u[0], (float)u[1], (float)u[2], (float)u[3]);
    }
    return make_float4(left > 0 ? (float)p[0] : 0.0f, left > 1 ? (float)p[1] : 0.0f, left > 2 ? (float)p[2] : 0.0f, left > 3 ? (float)p[3] : 0.0f);
}

template <class Ty> __device__ __forceinline__ void store4(typename Ty::T *p, int64_t left, bool wide, float4 v)
{
    typedef typename Ty::T T;
    T u[4] = {(T)v.x, (T)v.y, (T)v.z, (T)v.w};
    if (wide && left >= 4) {
        if constexpr (sizeof(T) == 4) __builtin_nontemporal_store(*(f4 *)u, (f4 *)p);
        else __builtin_nontemporal_store(*(i2 *)u, (i2 *)p);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < left) p[i] = u[i];
    }
}

template <class Ty> bool wide4(const void *p, int64_t stride)
{
    return (uintptr_t)p % (4 * sizeof(typename Ty::T)) == 0 && stride % 4 == 0;
}

template <class Y, class O> __global__ __launch_bounds__(256) void experts_sum_kernel(SumArgs a, bool wide_y, bool wide_o)
{
    const int k = a.order.k;
    for (int64_t t = blockIdx.x; t < a.order.T; t += gridDim.x)
        for (int64_t c = (int64_t)blockIdx.y * SPAN + threadIdx.x * 4; c < a.n; c += (int64_t)gridDim.y * SPAN) {
            float4 sum = make_float4(0, 0, 0, 0);
            for (int j = 0; j < k; j++) {
                const int place = a.order.places[t * k + j];
                if (place < 0) continue;
                const float w = a.weights ? a.weights[t * k + j] : 1.0f;
                const float4 v = load4<Y, true>((const typename Y::T *)a.y + (int64_t)place * a.y_stride + c, a.n - c, wide_y);
                sum.x = fmaf(w, v.x, sum.x);
                sum.y = fmaf(w, v.y, sum.y);
                sum.z = fmaf(w, v.z, sum.z);
                sum.w = fmaf(w, v.w, sum.w);
            }
            store4<O>((typename O::T *)a.out + t * a.stride + c, a.n - c, wide_o, sum);
        }
}

// One wave for each slot: a row of d_out is read once for each of its experts, from the caches but for the first time (they are neighbours, and d_out is
// read to be kept, y is not).
template <class Y, class O> __global__ __launch_bounds__(256) void experts_sum_backward_kernel(SumArgs a, bool wide_y, bool wide_o)
{
    const int k = a.order.k, lane = threadIdx.x & 63;
    const int64_t slots = a.order.T * k;
    for (int64_t s = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); s < slots; s += (int64_t)gridDim.x * 4) {
        const int64_t t = s / k;
        const int place = a.order.places[s];
        float sum = 0.0f;
        if (place >= 0)
            for (int64_t c = lane * 4; c < a.n; c += 256) {
                const float4 d = load4<O, false>((const typename O::T *)a.d_out + t * a.stride + c, a.n - c, wide_o);
                const float4 v = load4<Y, true>((const typename Y::T *)a.y + (int64_t)place * a.y_stride + c, a.n - c, wide_y);
                sum = fmaf(d.x, v.x, sum);
                sum = fmaf(d.y, v.y, sum);
                sum = fmaf(d.z, v.z, sum);
                sum = fmaf(d.w, v.w, sum);
            }
        sum = wave_sum(sum);
        if (lane == 0) a.d_weights[s] = sum;
    }
}

}  // namespace

hipError_t launch_experts_sum(const SumArgs &a, int y_type, int type, hipStream_t s)
{
    const int64_t spans = (a.n + SPAN - 1) / SPAN;
    const dim3 grid((unsigned)(a.order.T < (1 << 20) ? a.order.T : (1 << 20)), (unsigned)(spans < 8 ? spans : 8));
    return with_type(y_type, [&](auto y) {
        return with_type(type, [&](auto o) {
            experts_sum_kernel<decltype(y), decltype(o)><<<grid, 256, 0, s>>>(a, wide4<decltype(y)>(a.y, a.y_stride), wide4<decltype(o)>(a.out, a.stride));
            return hipGetLastError();
        });
    });
}

hipError_t launch_experts_sum_backward(const SumArgs &a, int y_type, int type, hipStream_t s)
{
    const int64_t rows = (a.order.T * a.order.k + 3) / 4;
    const unsigned grid = (unsigned)(rows < (1 << 20) ? rows : (1 << 20));
    return with_type(y_type, [&](auto y) {
        return with_type(type, [&](auto o) {
            experts_sum_backward_kernel<decltype(y), decltype(o)><<<grid, 256, 0, s>>>(a, wide4<decltype(y)>(a.y, a.y_stride), wide4<decltype(o)>(a.d_out, a.stride));
            return hipGetLastError();
        });
    });
}

}  // namespace asgd
