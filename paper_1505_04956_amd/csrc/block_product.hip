// Products of matrices in 8-bit blocks on the matrix cores (v_mfma_f32_16x16x128_f8f6f4: one instruction is one block of
// the contraction).  out^T = b a^T is what is formed: rows of b are the instruction's rows, rows of a its columns, so that a
// lane holds four neighbours of one row of out, and the scale of its row of a is one number a lane.
//
// The order of the 128 bytes of a block among the lanes is free as long as both operands have the same: lane l holds the
// sixteen bytes l / 16 and l / 16 + 4 of row l % 16.
#include <type_traits>

#include "experts_internal.h"

namespace asgd {

namespace {

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

// 64 lanes x 16 bytes, from an address of each lane to consecutive places of the LDS
__device__ __forceinline__ void to_lds(const uint8_t *from, uint8_t *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
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

// The expert whose rows the tile `tile` of `rows` places has, with every expert's first place at the begin of a tile; the
// tile's first place and the expert's end.  false: no such tile.  A wave does it, 64 experts at a time.
__device__ __forceinline__ bool tile_of_expert(const asgd_route_order &o, int64_t tile, int rows, int &expert, int64_t &first, int64_t &end)
{
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int e0 = 0; e0 < o.E; e0 += 64) {
        const int e = e0 + lane;
        const int begin = e < o.E ? o.offsets[e] : 0, stop = e < o.E ? o.offsets[e + 1] : 0;
        const int tiles = (stop - begin + rows - 1) / rows;
        int sum = tiles;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int u = __shfl_up(sum, m);
            if (lane >= m) sum += u;
        }
        const unsigned long long past = __ballot(before + sum > tile);
        if (past) {
            const int at = __ffsll((long long)past) - 1;
            expert = __builtin_amdgcn_readfirstlane(e0 + at);
            const int mine = __shfl(begin, at), last = __shfl(stop, at), done = __shfl(sum - tiles, at);
            first = __builtin_amdgcn_readfirstlane((int)(mine + (tile - before - done) * rows));
            end = __builtin_amdgcn_readfirstlane(last);
            return true;
        }
        before += __shfl(sum, 63);
    }
    return false;
}

// Workgroups go round the eight dies; each die gets a run of neighbouring tiles, whose operands its L2 then shares.
__device__ __forceinline__ int64_t tile_of_group(int64_t id, int64_t n)
{
    const int64_t die = id & 7, at = id >> 3, share = n >> 3, rest = n & 7;
    return die * share + (die < rest ? die : rest) + at;
}

// A tile of TOK rows of a and WT rows of b; the waves are TOK_WAVES x WT_WAVES.  A block of the contraction of both goes to
// the LDS (16-byte pieces of a row at their number xor the row's low bits: the lanes of a read then spread over the banks)
// while the block before it is multiplied.
template <int TOK, int WT, int TOK_WAVES, int WT_WAVES, bool SQUARES, bool EXACT, class Out>
__global__ __launch_bounds__(64 * TOK_WAVES * WT_WAVES) void product_kernel(ProductArgs p, int64_t tiles_tok, int64_t tiles_wt, bool wide)
{
    constexpr int WAVES = TOK_WAVES * WT_WAVES, J = TOK / TOK_WAVES / 16, I = WT / WT_WAVES / 16;
    constexpr int SEGMENTS = (TOK + WT) / 8 / WAVES;             // of eight rows, that a wave brings
    static_assert((TOK + WT) / 8 % WAVES == 0 && WT / WT_WAVES <= BLOCK8, "");
    __shared__ __align__(16) uint8_t stage0[(TOK + WT) * BLOCK8];
    __shared__ __align__(16) uint8_t stage1[(TOK + WT) * BLOCK8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_tok = wave % TOK_WAVES * (J * 16), wave_wt = wave / TOK_WAVES * (I * 16);

    // which tile: strips of eight tiles of a, all tiles of b for each
    const int64_t id = tile_of_group(blockIdx.x, gridDim.x);
    int64_t matrix = 0, within = id;
    if (p.mode == ASGD_PRODUCT_OVER) {
        matrix = id / (tiles_tok * tiles_wt);
        within = id - matrix * tiles_tok * tiles_wt;
    }
    const int64_t strip = within / (8 * tiles_wt), in_strip = within - strip * 8 * tiles_wt;
    const int64_t high = tiles_tok - strip * 8 < 8 ? tiles_tok - strip * 8 : 8;
    const int64_t tile_wt = in_strip / high, tile_tok = strip * 8 + in_strip - tile_wt * high;

    int64_t first = tile_tok * TOK, end = p.rows_a, k0 = 0, k1 = p.kb;
    const int64_t first_wt = tile_wt * WT;
    if (p.mode == ASGD_PRODUCT_GATHER || p.mode == ASGD_PRODUCT_PLACES) {
        int e;
        if (!tile_of_expert(p.order, tile_tok, TOK, e, first, end)) return;
        matrix = e;
    } else if (p.mode == ASGD_PRODUCT_OVER) {
        k0 = p.order.blocks[matrix];
        k1 = p.order.blocks[matrix + 1];
    }
    const int64_t row_bytes = p.kb * BLOCK8;
    const uint8_t *b = p.b + (p.mode == ASGD_PRODUCT_OVER ? 0 : matrix * p.rows_b * row_bytes);
    const auto row_of_a = [&](int64_t r) {                        // (rows beyond the last: the last again)
        r = r < end ? r : end - 1;
        return p.mode == ASGD_PRODUCT_GATHER ? (int64_t)(p.order.slots[r] / p.order.k) : r;
    };

    const uint8_t *from[SEGMENTS];
#pragma unroll
    for (int s = 0; s < SEGMENTS; s++) {
        const int row = (wave * SEGMENTS + s) * 8 + (lane >> 3), piece = (lane & 7) ^ (lane >> 3);
        if (row < TOK) from[s] = p.a + row_of_a(first + row) * row_bytes + piece * 16;
        else {
            const int64_t r = first_wt + row - TOK;
            from[s] = b + (r < p.rows_b ? r : p.rows_b - 1) * row_bytes + piece * 16;
        }
    }
    const auto bring = [&](int64_t kb, uint8_t *stage) {
#pragma unroll
        for (int s = 0; s < SEGMENTS; s++) to_lds(from[s] + kb * BLOCK8, stage + (wave * SEGMENTS + s) * 1024);
    };

    const float *scale_a[J];
#pragma unroll
    for (int j = 0; j < J; j++) scale_a[j] = p.sa + row_of_a(first + wave_tok + j * 16 + (lane & 15));
    int64_t square = 0;
    if (SQUARES) {
        const int64_t nb = blocks8(p.rows_b), at = (first_wt + wave_wt) / BLOCK8;
        square = (matrix * nb + (at < nb ? at : nb - 1)) * p.kb;
    }

    v4f sum[I][J];
#pragma unroll
    for (int i = 0; i < I; i++)
#pragma unroll
        for (int j = 0; j < J; j++) sum[i][j] = {0.0f, 0.0f, 0.0f, 0.0f};

    const int low = ((lane >> 4) ^ (lane & 7)) * 16, row_at = (lane & 15) * BLOCK8;
    const auto operand = [&](const uint8_t *stage, int row) {
        const uint8_t *at = stage + row * BLOCK8 + row_at;
        const v4i u = *(const v4i *)(at + low), v = *(const v4i *)(at + (low ^ 64));
        Operand<EXACT> o;
        o.set(u, v);
        return o;
    };
    const auto multiply = [&](int64_t kb, const uint8_t *stage) {
        float s[J];
        Operand<EXACT> a[J];
#pragma unroll
        for (int j = 0; j < J; j++) {
            s[j] = scale_a[j][kb * p.rows_a];
            a[j] = operand(stage, wave_tok + j * 16);
        }
        if (SQUARES) {
            const float sb = p.sb[square + kb];
#pragma unroll
            for (int j = 0; j < J; j++) s[j] *= sb;
        }
#pragma unroll
        for (int i = 0; i < I; i++) {
            const Operand<EXACT> w = operand(stage, TOK + wave_wt + i * 16);
            v4f sb;
            if (!SQUARES) {
                const int64_t r = first_wt + wave_wt + i * 16 + (lane >> 4) * 4;
#pragma unroll
                for (int n = 0; n < 4; n++) sb[n] = p.sb[kb * p.rows_b + (r + n < p.rows_b ? r + n : p.rows_b - 1)];
            }
#pragma unroll
            for (int j = 0; j < J; j++) {
                const v4f part = block_product(w, a[j]);
#pragma unroll
                for (int n = 0; n < 4; n++) {
                    const float v = SQUARES ? part[n] : part[n] * sb[n];
                    sum[i][j][n] = fmaf(v, s[j], sum[i][j][n]);
                }
            }
        }
    };

    if (k0 < k1) bring(k0, stage0);
    __syncthreads();
    for (int64_t kb = k0; kb < k1; kb += 2) {
        if (kb + 1 < k1) bring(kb + 1, stage1);
        multiply(kb, stage0);
        __syncthreads();
        if (kb + 1 >= k1) break;
        if (kb + 2 < k1) bring(kb + 2, stage0);
        multiply(kb + 1, stage1);
        __syncthreads();
    }

    typedef typename Out::T T;
    T *out = (T *)p.out + (p.mode == ASGD_PRODUCT_OVER ? matrix * p.rows_a * p.stride : 0);
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int64_t r = first + wave_tok + j * 16 + (lane & 15);
        if (r < end) {
#pragma unroll
            for (int i = 0; i < I; i++) {
                const int64_t c = first_wt + wave_wt + i * 16 + (lane >> 4) * 4;
                store_four<Out>(out + r * p.stride + c, p.rows_b - c, wide, sum[i][j]);
            }
        }
    }
}

// ---- few rows, not in 8 bits yet --------------------------------------------------------------------------------------
// What counts is that the weights arrive: they go from memory to registers, sixteen rows of one block of 128 a wave and
// instruction, and the eight waves of a workgroup share the blocks of the contraction of sixteen rows of b.  The rows of a are
// brought to 8 bits in the registers of the lanes that need them.
constexpr int RAW_WAVES = 8;

template <class Ty> __device__ __forceinline__ void raw_block(const typename Ty::T *row, bool there, bool wide, int64_t c, int64_t cols, float &scale, v4i &lo, v4i &hi)
{
    typedef typename Ty::T T;
    float v[32];
    if (there && wide && c + 32 <= cols) {
        T u[32];
#pragma unroll
        for (int n = 0; n < (int)(32 * sizeof(T) / 16); n++) *((uint4 *)u + n) = *((const uint4 *)(row + c) + n);
#pragma unroll
        for (int i = 0; i < 32; i++) v[i] = (float)u[i];
    } else {
#pragma unroll
        for (int i = 0; i < 32; i++) v[i] = there && c + i < cols ? (float)row[c + i] : 0.0f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 32; i++) top = max(top, magnitude_bits(v[i]));
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

// grid: strips of sixteen rows of b, and (GATHER) places
template <class In, bool EXACT, class Out> __global__ __launch_bounds__(64 * RAW_WAVES) void product_raw_kernel(ProductArgs p, bool wide_in, bool wide)
{
    __shared__ float parts[RAW_WAVES][64][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t strip = blockIdx.x;
    int64_t matrix = 0, first = 0, end = p.rows_a;
    if (p.mode == ASGD_PRODUCT_GATHER) {
        int e;
        if (!tile_of_expert(p.order, blockIdx.y, 1, e, first, end)) return;
        matrix = e;
        end = first + 1;
    }
    const int tok = lane & 15, quarter = lane >> 4;
    const bool there = first + tok < end;
    const int64_t src = !there ? 0 : p.mode == ASGD_PRODUCT_GATHER ? p.order.slots[first + tok] / p.order.k : first + tok;
    const typename In::T *row = (const typename In::T *)p.a + src * p.stride_raw;
    const int64_t r = strip * 16 + tok, row_bytes = p.kb * BLOCK8;
    const uint8_t *b = p.b + (matrix * p.rows_b + (r < p.rows_b ? r : p.rows_b - 1)) * row_bytes + quarter * 32;
    const float *sb = p.sb + (matrix * blocks8(p.rows_b) + strip / 8) * p.kb;
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t kb = wave; kb < p.kb; kb += RAW_WAVES) {
        const v4i u = *(const v4i *)(b + kb * BLOCK8), v = *(const v4i *)(b + kb * BLOCK8 + 16);
        float scale;
        v4i lo, hi;
        raw_block<In>(row, there, wide_in, kb * BLOCK8 + quarter * 32, p.cols, scale, lo, hi);
        scale *= sb[kb];
        Operand<EXACT> w, a;
        w.set(u, v);
        a.set(lo, hi);
        const v4f part = block_product(w, a);
#pragma unroll
        for (int n = 0; n < 4; n++) sum[n] = fmaf(part[n], scale, sum[n]);
    }
    *(v4f *)parts[wave][lane] = sum;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < RAW_WAVES; w++) sum += *(v4f *)parts[w][lane];
        const int64_t c = strip * 16 + quarter * 4;
        if (there) store_four<Out>((typename Out::T *)p.out + (first + tok) * p.stride + c, p.rows_b - c, wide, sum);
    }
}

}  // namespace

hipError_t launch_product(const ProductArgs &p, bool squares, int type, hipStream_t s)
{
    constexpr int TOK = 128, WT = 128;
    const int64_t tiles_wt = (p.rows_b + WT - 1) / WT;
    int64_t tiles_tok = (p.rows_a + TOK - 1) / TOK, tiles = tiles_tok * tiles_wt;
    if (p.mode == ASGD_PRODUCT_GATHER || p.mode == ASGD_PRODUCT_PLACES) {
        const int64_t slots = p.order.T * p.order.k;
        tiles_tok = slots / TOK + (slots < p.order.E ? slots : p.order.E);
        tiles = tiles_tok * tiles_wt;
    } else if (p.mode == ASGD_PRODUCT_OVER) tiles *= p.order.E;
    const bool wide = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * type_size(type)) == 0;
    return with_type(type, [&](auto out) {
        const auto go = [&](auto sq, auto exact) {
            product_kernel<TOK, WT, 2, 2, decltype(sq)::value, decltype(exact)::value, decltype(out)><<<(unsigned)tiles, 256, 0, s>>>(p, tiles_tok, tiles_wt, wide);
            return hipGetLastError();
        };
        const std::true_type yes;
        const std::false_type no;
        return squares ? p.exact ? go(yes, yes) : go(yes, no) : p.exact ? go(no, yes) : go(no, no);
    });
}

hipError_t launch_product_raw(const ProductArgs &p, int raw_type, int type, hipStream_t s)
{
    const bool wide = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * type_size(type)) == 0;
    const bool wide_in = p.stride_raw * (int64_t)type_size(raw_type) % 16 == 0 && ((uintptr_t)p.a & 15) == 0;
    const dim3 grid((unsigned)((p.rows_b + 15) / 16), p.mode == ASGD_PRODUCT_GATHER ? (unsigned)(p.order.T * p.order.k) : 1u);
    return with_type(raw_type, [&](auto in) {
        return with_type(type, [&](auto out) {
            if (p.exact) product_raw_kernel<decltype(in), true, decltype(out)><<<grid, 64 * RAW_WAVES, 0, s>>>(p, wide_in, wide);
            else product_raw_kernel<decltype(in), false, decltype(out)><<<grid, 64 * RAW_WAVES, 0, s>>>(p, wide_in, wide);
            return hipGetLastError();
        });
    });
}

}  // namespace asgd
