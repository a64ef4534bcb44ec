// To 4 bits in blocks of 32, and back.  Both read their input once and write their result once, and memory bounds them: 16384 x 4096 in bfloat16, 134 MB, to 4 bits
// 35 us (4.8 TB/s), back 40 (4.2; a large copy reaches 4.9).
#include "four_bits.h"

namespace asgd {

namespace {

// Four lanes take a block, eight elements each; 32 lanes a run of 256 columns, a wave two of them next to each other.
template <class Ty> __global__ __launch_bounds__(256) void quantize_four_kernel(FourArgs q, int64_t groups)
{
    typedef typename Ty::T T;
    const int64_t runs = runs4(q.cols);
    const int part = threadIdx.x & 31;
    for (int64_t g = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); g < groups; g += (int64_t)gridDim.x * 8) {
        const int64_t r = g / runs, run = g - r * runs, c = run * RUN4 + part * 8;
        float v[8];
        eight_of((const T *)q.x + r * q.stride, c, q.cols, v);
        uint32_t scale;
        *(uint32_t *)(q.values + g * RUN4_BYTES + part * 4) = Parts<4>::to(v, scale);
        Parts<4>::put_scale(q.scales + g * RUN4_SCALES, part, scale);
    }
}

// A thread takes eight values.
template <class Ty> __global__ __launch_bounds__(256) void expand_four_kernel(FourArgs q, int64_t groups)
{
    typedef typename Ty::T T;
    const int64_t runs = runs4(q.cols);
    const int part = threadIdx.x & 31;
    for (int64_t g = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); g < groups; g += (int64_t)gridDim.x * 8) {
        const int64_t r = g / runs, run = g - r * runs, c = run * RUN4 + part * 8;
        if (c >= q.cols) continue;
        const uint32_t u = *(const uint32_t *)(q.values + g * RUN4_BYTES + part * 4), byte = q.scales[g * RUN4_SCALES + (part >> 2)];
        const float s = byte == 255 ? __uint_as_float(0x7FC00000u) : byte ? four_scale_value(byte) : __uint_as_float(0x00400000u);
        Eight<T> o;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t m = u >> (4 * i) & 7;
            // 0, 0.5, then (1 + low bit / 2) * 2^(high bits - 1)
            const float a = m < 2 ? 0.5f * (float)m : __uint_as_float((126u + (m >> 1)) << 23 | (m & 1) << 22);
            o.v[i] = (T)((u >> (4 * i) & 8 ? -a : a) * s);
        }
        T *p = (T *)const_cast<void *>(q.x) + r * q.stride + c;
        if (c + 8 <= q.cols) *(Eight<T> *)p = o;
        else
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (c + i < q.cols) p[i] = o.v[i];
    }
}

unsigned grid_of(int64_t groups) { return (unsigned)((groups + 7) / 8 < (1 << 20) ? (groups + 7) / 8 : 1 << 20); }

}  // namespace

hipError_t launch_quantize_four(const FourArgs &q, int type, hipStream_t s)
{
    const int64_t groups = q.rows * runs4(q.cols);
    return with_type(type, [&](auto ty) {
        quantize_four_kernel<decltype(ty)><<<grid_of(groups), 256, 0, s>>>(q, groups);
        return hipGetLastError();
    });
}

hipError_t launch_expand_four(const FourArgs &q, int type, hipStream_t s)
{
    const int64_t groups = q.rows * runs4(q.cols);
    return with_type(type, [&](auto ty) {
        expand_four_kernel<decltype(ty)><<<grid_of(groups), 256, 0, s>>>(q, groups);
        return hipGetLastError();
    });
}

}  // namespace asgd
