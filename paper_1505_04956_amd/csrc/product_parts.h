// What the products' kernels share: operands in 8 bits, loads to the LDS, stores of results, which expert's rows a tile has.
#pragma once

#include <type_traits>

#include "experts_internal.h"

namespace asgd {

namespace {

template <int N> using One = std::integral_constant<int, N>;

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// A lane's part of sixteen rows of one block: as it is, or (exact) as 16-bit numbers, which hold every e4m3 number.
template <bool EXACT> struct Operand;
template <> struct Operand<false> {
    v8i v;
    __device__ __forceinline__ void set(v4i u, v4i w) { v = (v8i){u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]}; }
};
template <> struct Operand<true> {
    v8h v[4];
    __device__ __forceinline__ void set(v4i u, v4i w)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int lo = i < 2 ? u[2 * i] : w[2 * i - 4], hi = i < 2 ? u[2 * i + 1] : w[2 * i - 3];
            const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
            const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
            v[i] = (v8h){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
        }
    }
};

// The sums of a block's products.  The 8-bit instruction adds eight neighbouring products at a time after aligning them to the largest
// and drops what lies more than 14 bits below it (measured: a product of 4 beside one of 448 * 448 is lost among the eight, kept
// anywhere else), an error of 1.5e-5 (normal values) to 7e-5 (values over six octaves) of the result; the 16-bit one, 3e-7.
__device__ __forceinline__ v4f block_product(const Operand<false> &a, const Operand<false> &b)
{
    const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, zero, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ v4f block_product(const Operand<true> &a, const Operand<true> &b)
{
    v4f part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; i++) part = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v[i], b.v[i], part, 0, 0, 0);
    return part;
}

// 64 lanes x 16 bytes, from a base and an offset of each lane to consecutive places of the LDS; and 64 x 4 bytes
template <class Offset> __device__ __forceinline__ void to_lds(const uint8_t *base, Offset offset, uint8_t *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + offset),
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
template <class Offset> __device__ __forceinline__ void to_lds4(const uint8_t *base, Offset offset, uint8_t *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + offset),
                                     (__attribute__((address_space(3))) void *)to, 4, 0, 0);
}

template <class Ty> __device__ __forceinline__ void store_four(typename Ty::T *p, int64_t left, bool wide, v4f v)
{
    typedef typename Ty::T T;
    if (wide && left >= 4) {
        T u[4] = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        if constexpr (sizeof(T) == 4) *(uint4 *)p = *(uint4 *)u;
        else *(uint2 *)p = *(uint2 *)u;
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < left) p[i] = (T)v[i];
    }
}

// sixteen bytes of a row, of which `left` elements exist; wide: rows begin at a multiple of 16 bytes.  They pass by the second cache, whose
// place belongs to the operands (65536 x 1024 x 128 to float32, bringing a to 8 bits included: 61 us; kept there, 65; gradients of 64 experts' weights of
// 2048 x 2048 306 and 395; the sum of experts that reads 129 MB of them next loses nothing by it)
template <class T> __device__ __forceinline__ void store16(T *p, int64_t left, bool wide, v4i v)
{
    constexpr int N = 16 / sizeof(T);
    if (wide && left >= N) __builtin_nontemporal_store(v, (v4i *)p);
    else {
        T u[N];
        *(v4i *)u = v;
#pragma unroll
        for (int i = 0; i < N; i++)
            if (i < left) p[i] = u[i];
    }
}

// The expert whose rows the tile `tile` of `rows` places has, with every expert's first place at the begin of a tile; the
// tile's first place and the expert's end.  false: no such tile.  A wave does it, 64 experts at a time.
__device__ __forceinline__ bool tile_of_expert(const asgd_route_order &o, int64_t tile, int rows, int &expert, int64_t &first, int64_t &end)
{
    const int lane = threadIdx.x & 63;
    int before = 0, begin = o.offsets[min(lane, o.E)], stop = o.offsets[min(lane + 1, o.E)];
    for (int e0 = 0; e0 < o.E; e0 += 64) {
        const int from = begin, to = stop;
        if (e0 + 64 < o.E) {                                      // (the next are on their way meanwhile)
            begin = o.offsets[min(e0 + 64 + lane, o.E)];
            stop = o.offsets[min(e0 + 65 + lane, o.E)];
        }
        const int tiles = (int)((unsigned)(to - from + rows - 1) / (unsigned)rows), sum = wave_scan(tiles);
        const unsigned long long past = __ballot(before + sum > (int)tile);
        if (past) {
            const int at = __ffsll((long long)past) - 1, done = before + __builtin_amdgcn_readlane(sum - tiles, at);
            expert = e0 + at;
            first = __builtin_amdgcn_readlane(from, at) + ((int)tile - done) * rows;
            end = __builtin_amdgcn_readlane(to, at);
            return true;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// The same for tiles of 128 places, whose number before each expert the order holds.
__device__ __forceinline__ bool block_of_expert(const asgd_route_order &o, int tile, int &expert, int64_t &first, int64_t &end)
{
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < o.E; e0 += 64) {
        const int e = e0 + lane < o.E ? e0 + lane : o.E - 1;
        const int stop = o.blocks[e + 1], begin = o.blocks[e], place = o.offsets[e], last = o.offsets[e + 1];
        const unsigned long long past = __ballot(stop > tile);
        if (past) {
            const int at = __ffsll((long long)past) - 1;
            expert = e0 + at;
            first = __builtin_amdgcn_readlane(place, at) + (tile - __builtin_amdgcn_readlane(begin, at)) * BLOCK8;
            end = __builtin_amdgcn_readlane(last, at);
            return true;
        }
    }
    return false;
}

// Workgroups go round the eight dies; each die gets a run of neighbouring tiles, whose operands its L2 then shares.
__device__ __forceinline__ uint32_t tile_of_group(uint32_t id, uint32_t n)
{
    const uint32_t die = id & 7, at = id >> 3, share = n >> 3, rest = n & 7;
    return die * share + (die < rest ? die : rest) + at;
}

// a lane's 32 elements of a block of a row: fetched early, brought to 8 bits when they are there
template <class Ty> struct RawBlock {
    typename Ty::T u[32];
    __device__ __forceinline__ void load(const typename Ty::T *row, bool there, bool wide, int64_t c, int64_t cols)
    {
        if (wide && c + 32 <= cols) {
            if (there)
#pragma unroll
                for (int n = 0; n < (int)(32 * sizeof(typename Ty::T) / 16); n++) *((uint4 *)u + n) = *((const uint4 *)(row + c) + n);
        } else
#pragma unroll
            for (int i = 0; i < 32; i++) u[i] = there && c + i < cols ? row[c + i] : (typename Ty::T)0.0f;
    }
    __device__ __forceinline__ void set(bool there, float &scale, v4i &lo, v4i &hi) const
    {
        float v[32];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 32; i++) {
            v[i] = there ? (float)u[i] : 0.0f;
            top = max(top, magnitude_bits(v[i]));
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        float inverse;
        block_scale(top, scale, inverse);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            lo[i] = (int)eight_bits(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], inverse);
            hi[i] = (int)eight_bits(v[4 * i + 16], v[4 * i + 17], v[4 * i + 18], v[4 * i + 19], inverse);
        }
    }
};
template <> struct RawBlock<void> {};

}  // namespace

}  // namespace asgd
