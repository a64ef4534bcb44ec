// 4-bit floating point (e2m1) in blocks of 32 with a power of two as scale: what the kernels that make or multiply it share.
#pragma once

#include "product_parts.h"

namespace asgd {

constexpr int BLOCK4 = 32;                // columns that share a scale
constexpr int RUN4 = 256;                 // columns of a row that are laid out together: 128 bytes of values, 8 of scales
constexpr int RUN4_BYTES = RUN4 / 2, RUN4_SCALES = RUN4 / BLOCK4;

__host__ __device__ inline int64_t runs4(int64_t cols) { return (cols + RUN4 - 1) / RUN4; }

namespace {

// The byte of the scale of a block whose largest magnitude has these bits: one more where the first bit after the leading one and the next are set (1.75 and
// more), so that the block's largest value rounds to 4 times the larger scale and not to 6 times the smaller.
__device__ __forceinline__ uint32_t four_scale(uint32_t top)
{
    if (top >= 0x7F800000u) return 255u;
    const int e = (int)((top + (1u << 21)) >> 23) - 2;
    return (uint32_t)min(max(e, 1), 252);
}
__device__ __forceinline__ float four_scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }      // (255: infinity, times which nothing is a number)

// eight values to 4 bits, the first in the lowest; v / scale to nearest even, cut at 6
__device__ __forceinline__ uint32_t four_bits(const float *v, float scale)
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
}

// eight elements at any address that an element may have
template <class T> struct Eight { T v[8]; } __attribute__((packed));

// elements c .. c + 7 of a row of cols
template <class T> __device__ __forceinline__ void eight_of(const T *row, int64_t c, int64_t cols, float (&v)[8])
{
    if (c + 8 <= cols) {
        const Eight<T> u = *(const Eight<T> *)(row + c);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = (float)u.v[i];
    } else
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = c + i < cols ? (float)row[c + i] : 0.0f;
}

// To 8 or 4 bits, eight neighbours a lane: sixteen lanes take a block of 128 columns in 8 bits, 32 lanes a run of 256 in 4 bits; either is 128 bytes and its scales.
template <int BITS> struct Parts;
template <> struct Parts<8> {
    static constexpr int LANES = 16, BYTES = 8;
    typedef uint2 Bytes;
    typedef float Scale;
    static __device__ __forceinline__ Bytes to(const float (&v)[8], Scale &scale)
    {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) top = max(top, magnitude_bits(v[i]));
        float inverse;
        block_scale((uint32_t)row_max((int)top), scale, inverse);
        return make_uint2(eight_bits(v[0], v[1], v[2], v[3], inverse), eight_bits(v[4], v[5], v[6], v[7], inverse));
    }
    static __device__ __forceinline__ void put_scale(uint8_t *scales, int part, Scale scale) { if (part == 0) *(float *)scales = scale; }
    static constexpr int SCALES = 4;             // bytes of a step
};
template <> struct Parts<4> {
    static constexpr int LANES = 32, BYTES = 4;
    typedef uint32_t Bytes;
    typedef uint32_t Scale;
    static __device__ __forceinline__ Bytes to(const float (&v)[8], Scale &scale)
    {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) top = max(top, magnitude_bits(v[i]));
        top = max(top, (uint32_t)across<XOR1>((int)top));
        top = max(top, (uint32_t)across<XOR2>((int)top));
        scale = four_scale(top);
        return four_bits(v, four_scale_value(scale));
    }
    static __device__ __forceinline__ void put_scale(uint8_t *scales, int part, Scale scale) { if ((part & 3) == 0) scales[part >> 2] = (uint8_t)scale; }
    static constexpr int SCALES = 8;
};

// sixteen rows of b (a lane's 32 columns of row lane % 16, columns lane / 16 * 32 of 128) times sixteen of a, added to `sum`, in which a lane has
// rows lane / 16 * 4 + i of b and row lane % 16 of a.  Scales: the bytes of the lane's own blocks.
__device__ __forceinline__ v4f four_product(v4i b, uint32_t scale_b, v4i a, uint32_t scale_a, v4f sum)
{
    const v8i u = {b[0], b[1], b[2], b[3], 0, 0, 0, 0}, w = {a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, w, sum, 4, 4, 0, (int)scale_b, 0, (int)scale_a);
}

}  // namespace

}  // namespace asgd
