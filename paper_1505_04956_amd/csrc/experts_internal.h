// Internal declarations of the routed experts: routing, products in 8-bit blocks, sums of a row's experts.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "asgd.h"

namespace asgd {

constexpr int BLOCK8 = 128;               // elements of the contraction that share a scale
constexpr float LARGEST8 = 448.0f;        // of e4m3
constexpr float SMALLEST8 = 1.0e-30f;     // magnitude a block is scaled as if it had, if it has less: keeps both factors normal numbers

__host__ __device__ inline int64_t blocks8(int64_t n) { return (n + BLOCK8 - 1) / BLOCK8; }

// Element types of the operands: loads and stores of one element as 32-bit float (one rounding, to nearest even).
struct F32 { typedef float T; static constexpr int type = ASGD_TYPE_F32; };
struct BF16 { typedef __bf16 T; static constexpr int type = ASGD_TYPE_BF16; };
struct F16 { typedef _Float16 T; static constexpr int type = ASGD_TYPE_F16; };

// f(BF16{}), f(F16{}) or f(F32{}) by ASGD_TYPE_* (checked before)
template <class F> inline auto with_type(int type, F f)
{
    if (type == ASGD_TYPE_BF16) return f(BF16{});
    if (type == ASGD_TYPE_F16) return f(F16{});
    return f(F32{});
}

inline size_t type_size(int type) { return type == ASGD_TYPE_F32 ? 4 : 2; }

// ---- launchers (arguments checked by the entry points) ---------------------------------------------------------
struct RouteArgs {
    const void *logits;
    const float *bias;
    const int32_t *ids_in;        // backward
    const float *d_weights;       // backward
    void *d_logits;               // backward
    int32_t *ids;
    float *weights;
    int64_t T, stride, d_stride;
    int E;
    asgd_route_rule rule;
};
hipError_t launch_route(const RouteArgs &a, int type, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs &a, int type, hipStream_t s);
size_t route_plan_bytes(int64_t slots, int E);
hipError_t launch_route_plan(const int32_t *ids, const asgd_route_order &o, void *work, hipStream_t s);

struct QuantArgs {
    const void *x;
    int64_t rows, cols, stride;   // of x
    int count;
    uint8_t *values;
    float *scales;
    int64_t out_rows, out_blocks; // of the result
    asgd_route_order order;       // (offsets null: none)
    const float *weights;
};
hipError_t launch_quantize_rows(const QuantArgs &q, int type, hipStream_t s);
hipError_t launch_quantize_turned(const QuantArgs &q, int type, hipStream_t s);
hipError_t launch_quantize_both(const QuantArgs &q, const asgd_blocks &rows, int type, hipStream_t s);
hipError_t launch_quantize_squares(const QuantArgs &q, int type, bool turned, hipStream_t s);

struct ProductArgs {
    const uint8_t *a, *b;
    const float *sa, *sb;
    int64_t rows_a, rows_b;       // rows of a (out's rows but where gathered), rows of one matrix of b
    int64_t kb;                   // blocks of the contraction
    int64_t stride_raw, cols;     // a in `raw_type`
    void *out;
    int64_t stride;
    asgd_route_order order;
    int mode;
    int exact;
};
int product_form(const ProductArgs &p, bool squares);      // ASGD_PRODUCT_FORM_* that launch_product() takes
hipError_t launch_product(const ProductArgs &p, bool squares, int type, hipStream_t s);
hipError_t launch_product_direct(const ProductArgs &p, const int32_t *ids, const float *weights, int k, int E, int raw_type, int type, hipStream_t s);
hipError_t launch_product_raw(const ProductArgs &p, int raw_type, int type, hipStream_t s);

// 4 bits: x, rows of cols elements `stride` apart, to values and scales; or back, x written
struct FourArgs {
    const void *x;
    int64_t rows, cols, stride;
    uint8_t *values, *scales;
};
hipError_t launch_quantize_four(const FourArgs &q, int type, hipStream_t s);
hipError_t launch_expand_four(const FourArgs &q, int type, hipStream_t s);
// (kb counts runs of 256 columns; sa and sb are bytes)
int product_four_form(const ProductArgs &p);
hipError_t launch_product_four(const ProductArgs &p, int type, hipStream_t s);
hipError_t launch_product_four_raw(const ProductArgs &p, int raw_type, int type, hipStream_t s);

struct LayerArgs {
    const void *x;
    int64_t x_stride, D, H, N;
    int x_type, T, k, E, activation;
    asgd_blocks up, down;
    int32_t *ids;
    float *weights;
    void *out;
    int64_t out_stride;
    bool wide_out;
};
size_t layer_bytes(int64_t T, int k, int64_t E, int64_t D, int64_t H);
hipError_t launch_layer(const LayerArgs &a, const RouteArgs &r, int logits_type, int type, void *work, hipStream_t s);
struct DirectArgs {               // x's rows of K columns times matrices of N rows in 4 bits
    const void *x;
    int64_t x_stride, K, N;
    int T, k, E;
    const int32_t *ids;
    const float *weights;
    asgd_blocks w;
    void *out;
    int64_t out_stride;
    bool wide_out;
};
hipError_t launch_direct_four(const DirectArgs &a, int x_type, int type, hipStream_t s);

struct SumArgs {
    const void *y, *d_out;
    int64_t n, y_stride, stride;
    asgd_route_order order;
    const float *weights;
    float *d_weights;
    void *out;
};
hipError_t launch_experts_sum(const SumArgs &a, int y_type, int type, hipStream_t s);
hipError_t launch_experts_sum_backward(const SumArgs &a, int y_type, int type, hipStream_t s);

// ---- device helpers --------------------------------------------------------------------------------------------
// Across lanes with the instruction that does the arithmetic (DPP); a lane the pattern leaves out keeps `old`.
template <int PATTERN, int ROWS = 0xF> __device__ __forceinline__ float from_lane(float old, float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), PATTERN, ROWS, 0xF, false));
}
constexpr int XOR1 = 0xB1, XOR2 = 0x4E, MIRROR8 = 0x141, MIRROR16 = 0x140, LANE15 = 0x142, LANE31 = 0x143;

// a pattern that leaves no lane out
template <int PATTERN> __device__ __forceinline__ float across(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), PATTERN, 0xF, 0xF, true)); }
template <int PATTERN> __device__ __forceinline__ int across(int v) { return __builtin_amdgcn_mov_dpp(v, PATTERN, 0xF, 0xF, true); }

// a number as an integer of the same order (minus zero before zero), and back
__device__ __forceinline__ int as_integer(float v) { return __float_as_int(v) ^ (__float_as_int(v) >> 31 & 0x7FFFFFFF); }
__device__ __forceinline__ float as_number(int v) { return __int_as_float(v ^ (v >> 31 & 0x7FFFFFFF)); }

// The largest, in all lanes (each step joins two halves that hold one value each, so a mirror does for an exchange).  Of integers a
// step is one instruction; of floats it would be four, since operands that may be signalling are made quiet first.
__device__ __forceinline__ int row_max(int v)                     // over sixteen lanes
{
    v = max(v, across<XOR1>(v));
    v = max(v, across<XOR2>(v));
    v = max(v, across<MIRROR8>(v));
    return max(v, across<MIRROR16>(v));
}
__device__ __forceinline__ int wave_max(int v)
{
    v = row_max(v);
    v = max(v, __builtin_amdgcn_update_dpp((int)0x80000000, v, LANE15, 0xA, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp((int)0x80000000, v, LANE31, 0xC, 0xF, false));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ float wave_max(float v) { return as_number(wave_max(as_integer(v))); }
__device__ __forceinline__ float wave_sum(float v)
{
    v += from_lane<XOR1>(0.0f, v);
    v += from_lane<XOR2>(0.0f, v);
    v += from_lane<MIRROR8>(0.0f, v);
    v += from_lane<MIRROR16>(0.0f, v);
    v += from_lane<LANE15, 0xA>(0.0f, v);
    v += from_lane<LANE31, 0xC>(0.0f, v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// a lane's sum with all lanes before it
__device__ __forceinline__ int wave_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);      // from one lane before, in a row of sixteen; two; four; eight
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, LANE15, 0xA, 0xF, false);
    return v + __builtin_amdgcn_update_dpp(0, v, LANE31, 0xC, 0xF, false);
}

// magnitude as an order-preserving integer: infinities and what is not a number are larger than all finite ones
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// scale and its inverse of a block whose largest magnitude has these bits
__device__ __forceinline__ void block_scale(uint32_t top, float &scale, float &inverse)
{
    if (top >= 0x7F800000u) {
        scale = __uint_as_float(0x7FC00000u);
        inverse = 0.0f;                       // (infinity times this is not a number: see eight_bits)
    } else {
        const float m = fmaxf(__uint_as_float(top), SMALLEST8);
        scale = m * (1.0f / LARGEST8);
        inverse = LARGEST8 * (1.0f / m);
    }
}
// four values to e4m3: v * inverse (one rounding), cut at the largest number, to nearest even.  The median of three is -448 where its
// first operand is not a number, so every byte is one of a number
__device__ __forceinline__ uint32_t eight_bits(float a, float b, float c, float d, float inverse)
{
    const float q0 = __builtin_amdgcn_fmed3f(a * inverse, -LARGEST8, LARGEST8), q1 = __builtin_amdgcn_fmed3f(b * inverse, -LARGEST8, LARGEST8);
    const float q2 = __builtin_amdgcn_fmed3f(c * inverse, -LARGEST8, LARGEST8), q3 = __builtin_amdgcn_fmed3f(d * inverse, -LARGEST8, LARGEST8);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(q0, q1, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q2, q3, r, true);
}

}  // namespace asgd
