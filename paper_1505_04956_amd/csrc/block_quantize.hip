// To 8 bits in blocks of 128: rows, the transpose's rows, both, squares.  With m the largest magnitude of a block (at least 1e-30) its scale is
// m * (1 / 448) and an element v becomes e4m3(v * (448 * (1 / m))), every operation rounded.  All read x once and write a byte an element (both: two), so memory
// bounds them; the largest magnitude of a block is found among the lanes that hold it.  8192 x 8192 in bfloat16: rows 38 us (5.3 TB/s),
// transpose 38 (5.3), both 64 (4.2), squares 34 (5.9), transposed 42 (4.8).  (A large copy reaches 4.7; part of x stays in the last cache.)
#include "experts_internal.h"

namespace asgd {

namespace {

// eight consecutive elements of a row; `left` of them exist, `wide`: all rows begin at a multiple of 16 bytes
template <class Ty> __device__ __forceinline__ void load8(const typename Ty::T *p, int64_t left, bool wide, float (&v)[8])
{
    typedef typename Ty::T T;
    if (wide && left >= 8) {
        T u[8];
        *(uint4 *)u = *(const uint4 *)p;
        if constexpr (sizeof(T) == 4) *((uint4 *)u + 1) = *((const uint4 *)p + 1);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = (float)u[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < left ? (float)p[i] : 0.0f;
    }
}

// Sixteen lanes take a block, eight elements each; the lanes of a wave take four blocks of one row next to each other.
template <class Ty> __global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs q, int64_t groups, bool wide)
{
    typedef typename Ty::T T;
    const int64_t kb = q.out_blocks;
    const int part = threadIdx.x & 15;
    for (int64_t g = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); g < groups; g += (int64_t)gridDim.x * 16) {
        const int64_t r = g / kb, b = g - r * kb;
        int64_t src = r;
        float w = 1.0f;
        bool there = true;
        if (q.order.slots) {
            const int slot = q.order.slots[r];
            there = slot >= 0;
            src = there ? slot / q.order.k : 0;
            if (q.weights && there) w = q.weights[slot];
        }
        if (!there) continue;                                      // (the sixteen lanes of a block go the same way)
        const int64_t c = b * BLOCK8 + part * 8;
        float v[8];
        load8<Ty>((const T *)q.x + src * q.stride + c, q.cols - c, wide, v);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (q.weights) v[i] *= w;
            top = max(top, magnitude_bits(v[i]));
        }
        top = (uint32_t)row_max((int)top);
        float scale, inverse;
        block_scale(top, scale, inverse);
        uint2 o;
        o.x = eight_bits(v[0], v[1], v[2], v[3], inverse);
        o.y = eight_bits(v[4], v[5], v[6], v[7], inverse);
        *(uint2 *)(q.values + (r * kb + b) * BLOCK8 + part * 8) = o;
        if (part == 0) q.scales[b * q.out_rows + r] = scale;
    }
}

// the expert whose blocks hold block rb: the last one that begins at or before it (and is not empty)
__device__ __forceinline__ int expert_of_block(const asgd_route_order &o, int64_t rb)
{
    int lo = 0, hi = o.E;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (o.blocks[mid] <= rb) lo = mid; else hi = mid;
    }
    return lo;
}

// The transpose: a workgroup takes 128 rows of x (a block of the result) and 64 columns (rows of the result).  A thread has eight
// neighbouring columns of four rows, so that loads are wide; it gives four neighbours of each of eight rows of the result, which go
// through the LDS to be written as whole lines.  (Two bytes a load, 8192 rows of 1024
// at 32768 places: 52 us; so, 24.)
template <class Ty> __global__ __launch_bounds__(256) void quantize_turned_kernel(QuantArgs q, bool wide)
{
    typedef typename Ty::T T;
    constexpr int PITCH = BLOCK8 + 4;
    __shared__ uint32_t tops[32][64];
    __shared__ uint32_t lines[64 * PITCH / 4];
    __shared__ int64_t source[BLOCK8];
    __shared__ float factor[BLOCK8];
    const int64_t rb = blockIdx.x;
    const int part = threadIdx.x & 7, rows = threadIdx.x >> 3;
    if (q.order.offsets) {
        if (rb >= q.order.blocks[q.order.E]) return;
        const int e = expert_of_block(q.order, rb);
        if (threadIdx.x < BLOCK8) {
            const int64_t p = q.order.offsets[e] + (rb - q.order.blocks[e]) * BLOCK8 + threadIdx.x;
            const bool there = p < q.order.offsets[e + 1];
            const int slot = there ? q.order.slots[p] : -1;
            source[threadIdx.x] = there ? slot / q.order.k : -1;
            factor[threadIdx.x] = there && q.weights ? q.weights[slot] : 1.0f;
        }
    } else if (threadIdx.x < BLOCK8) {
        const int64_t r = rb * BLOCK8 + threadIdx.x;
        source[threadIdx.x] = r < q.rows ? r : -1;
        factor[threadIdx.x] = 1.0f;
    }
    __syncthreads();
    for (int64_t cb = blockIdx.y; cb * 64 < q.cols; cb += gridDim.y) {
        const int64_t c = cb * 64 + part * 8;
        float v[4][8];
        uint32_t top[8] = {};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t r = source[rows * 4 + i];
            if (r >= 0) load8<Ty>((const T *)q.x + r * q.stride + c, q.cols - c, wide, v[i]);
            else
#pragma unroll
                for (int n = 0; n < 8; n++) v[i][n] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float w = q.weights ? factor[rows * 4 + i] : 1.0f;
#pragma unroll
            for (int n = 0; n < 8; n++) {
                if (q.weights) v[i][n] *= w;
                top[n] = max(top[n], magnitude_bits(v[i][n]));
            }
        }
        *(uint4 *)&tops[rows][part * 8] = make_uint4(top[0], top[1], top[2], top[3]);
        *(uint4 *)&tops[rows][part * 8 + 4] = make_uint4(top[4], top[5], top[6], top[7]);
        __syncthreads();
        if (threadIdx.x < 64) {
            uint32_t m = 0;
#pragma unroll
            for (int n = 0; n < 32; n++) m = max(m, tops[n][threadIdx.x]);
            float scale, inverse;
            block_scale(m, scale, inverse);
            if (cb * 64 + threadIdx.x < q.cols) q.scales[rb * q.out_rows + cb * 64 + threadIdx.x] = scale;
            tops[0][threadIdx.x] = __float_as_uint(inverse);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < 8; n++)
            lines[((part * 8 + n) * PITCH) / 4 + rows] = eight_bits(v[0][n], v[1][n], v[2][n], v[3][n], __uint_as_float(tops[0][part * 8 + n]));
        __syncthreads();
        const int line = threadIdx.x >> 2, quarter = threadIdx.x & 3;
        if (cb * 64 + line < q.cols) {
            const uint32_t *from = lines + line * (PITCH / 4) + quarter * 8;
            uint4 *to = (uint4 *)(q.values + ((cb * 64 + line) * q.out_blocks + rb) * BLOCK8 + quarter * 32);
            to[0] = make_uint4(from[0], from[1], from[2], from[3]);
            to[1] = make_uint4(from[4], from[5], from[6], from[7]);
        }
        __syncthreads();
    }
}

// Both at once, for training: the rows (of places) and the transpose, from one reading of x.  (8192 x 8192: 65 us, one after the other 39 and 38; with eight
// rows a thread, and half the waves, 78.)  A workgroup takes a square of 128 x 128, a thread eight neighbouring columns of four rows: sixteen lanes hold a row's block, 32 threads of different waves a column's.
template <class Ty> __global__ __launch_bounds__(512) void quantize_both_kernel(QuantArgs q, uint8_t *rows_values, float *rows_scales, int64_t rows_out, int64_t rows_blocks, bool wide)
{
    typedef typename Ty::T T;
    constexpr int PITCH = BLOCK8 + 4;
    __shared__ __align__(16) uint32_t tops[32][BLOCK8];
    __shared__ uint32_t lines[BLOCK8 * PITCH / 4];
    __shared__ int64_t source[BLOCK8], target[BLOCK8];
    __shared__ float factor[BLOCK8];
    const int64_t rb = blockIdx.x;
    const int part = threadIdx.x & 15, rows = threadIdx.x >> 4;
    if (q.order.offsets) {
        if (rb >= q.order.blocks[q.order.E]) return;
        const int e = expert_of_block(q.order, rb);
        if (threadIdx.x < BLOCK8) {
            const int64_t p = q.order.offsets[e] + (rb - q.order.blocks[e]) * BLOCK8 + threadIdx.x;
            const bool there = p < q.order.offsets[e + 1];
            const int slot = there ? q.order.slots[p] : -1;
            source[threadIdx.x] = there ? slot / q.order.k : -1;
            target[threadIdx.x] = p;
            factor[threadIdx.x] = there && q.weights ? q.weights[slot] : 1.0f;
        }
    } else if (threadIdx.x < BLOCK8) {
        const int64_t r = rb * BLOCK8 + threadIdx.x;
        source[threadIdx.x] = r < q.rows ? r : -1;
        target[threadIdx.x] = r;
        factor[threadIdx.x] = 1.0f;
    }
    __syncthreads();
    for (int64_t cb = blockIdx.y; cb * BLOCK8 < q.cols; cb += gridDim.y) {
        const int64_t c = cb * BLOCK8 + part * 8;
        float v[4][8];
        uint32_t top[8] = {};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t r = source[rows * 4 + i];
            if (r >= 0) load8<Ty>((const T *)q.x + r * q.stride + c, q.cols - c, wide, v[i]);
            else
#pragma unroll
                for (int n = 0; n < 8; n++) v[i][n] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int row = rows * 4 + i;
            uint32_t mine = 0;
#pragma unroll
            for (int n = 0; n < 8; n++) {
                if (q.weights) v[i][n] *= factor[row];
                const uint32_t m = magnitude_bits(v[i][n]);
                top[n] = max(top[n], m);
                mine = max(mine, m);
            }
            mine = (uint32_t)row_max((int)mine);
            float scale, inverse;
            block_scale(mine, scale, inverse);
            if (source[row] >= 0) {
                uint2 o;
                o.x = eight_bits(v[i][0], v[i][1], v[i][2], v[i][3], inverse);
                o.y = eight_bits(v[i][4], v[i][5], v[i][6], v[i][7], inverse);
                *(uint2 *)(rows_values + (target[row] * rows_blocks + cb) * BLOCK8 + part * 8) = o;
                if (part == 0) rows_scales[cb * rows_out + target[row]] = scale;
            }
        }
        *(uint4 *)&tops[rows][part * 8] = make_uint4(top[0], top[1], top[2], top[3]);
        *(uint4 *)&tops[rows][part * 8 + 4] = make_uint4(top[4], top[5], top[6], top[7]);
        __syncthreads();
        if (threadIdx.x < BLOCK8) {
            uint32_t m = 0;
#pragma unroll
            for (int n = 0; n < 32; n++) m = max(m, tops[n][threadIdx.x]);
            float scale, inverse;
            block_scale(m, scale, inverse);
            if (cb * BLOCK8 + threadIdx.x < q.cols) q.scales[rb * q.out_rows + cb * BLOCK8 + threadIdx.x] = scale;
            tops[0][threadIdx.x] = __float_as_uint(inverse);
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < 8; n++)
            lines[(part * 8 + n) * (PITCH / 4) + rows] = eight_bits(v[0][n], v[1][n], v[2][n], v[3][n], __uint_as_float(tops[0][part * 8 + n]));
        __syncthreads();
        const int line = threadIdx.x >> 2, quarter = threadIdx.x & 3;
        if (cb * BLOCK8 + line < q.cols) {
            const uint32_t *from = lines + line * (PITCH / 4) + quarter * 8;
            uint4 *to = (uint4 *)(q.values + ((cb * BLOCK8 + line) * q.out_blocks + rb) * BLOCK8 + quarter * 32);
#pragma unroll
            for (int n = 0; n < 2; n++) to[n] = make_uint4(from[4 * n], from[4 * n + 1], from[4 * n + 2], from[4 * n + 3]);
        }
        __syncthreads();
    }
}

// Squares: a workgroup of 256 takes one, a thread eight neighbouring columns of eight rows, which stay in registers until the largest of all is
// known.  (Read twice, the second time from the caches, an element a load: 116 us and transposed 184 for 8192 x 8192, where this takes 34 and 43.)
// The transposed square goes through the LDS to be written as whole lines.  Rows of the result beyond out_rows do not exist; columns
// beyond the data are zeros.
template <class Ty, bool TURNED> __global__ __launch_bounds__(256) void quantize_squares_kernel(QuantArgs q, bool wide)
{
    typedef typename Ty::T T;
    constexpr int PITCH = BLOCK8 + 4;
    __shared__ uint32_t tops[4];
    __shared__ uint32_t lines[TURNED ? BLOCK8 * PITCH / 4 : 1];
    const int part = threadIdx.x & 15, rows = threadIdx.x >> 4;
    const int64_t nb = blocks8(q.out_rows), kb = q.out_blocks, square = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (square >= nb * kb * q.count) return;
    const int64_t m = square / (nb * kb), ib = square / kb % nb, jb = square % kb;
    const T *x = (const T *)q.x + m * q.rows * q.stride;
    const int64_t r0 = (TURNED ? jb : ib) * BLOCK8 + rows * 8, c = (TURNED ? ib : jb) * BLOCK8 + part * 8;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (r0 + i < q.rows) load8<Ty>(x + (r0 + i) * q.stride + c, q.cols - c, wide, v[i]);
        else
#pragma unroll
            for (int n = 0; n < 8; n++) v[i][n] = 0.0f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
        for (int n = 0; n < 8; n++) top = max(top, magnitude_bits(v[i][n]));
    top = (uint32_t)wave_max((int)top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    float scale, inverse;
    block_scale(top, scale, inverse);
    if (threadIdx.x == 0) q.scales[square] = scale;
    uint8_t *out = q.values + (m * q.out_rows * kb + jb) * BLOCK8;
    if constexpr (TURNED) {
#pragma unroll
        for (int n = 0; n < 8; n++) {
            lines[(part * 8 + n) * (PITCH / 4) + rows * 2] = eight_bits(v[0][n], v[1][n], v[2][n], v[3][n], inverse);
            lines[(part * 8 + n) * (PITCH / 4) + rows * 2 + 1] = eight_bits(v[4][n], v[5][n], v[6][n], v[7][n], inverse);
        }
        __syncthreads();
        const int line = threadIdx.x >> 1, half = threadIdx.x & 1;
        if (ib * BLOCK8 + line < q.out_rows) {
            const uint32_t *from = lines + line * (PITCH / 4) + half * 16;
            uint4 *to = (uint4 *)(out + (ib * BLOCK8 + line) * kb * BLOCK8 + half * 64);
#pragma unroll
            for (int n = 0; n < 4; n++) to[n] = make_uint4(from[4 * n], from[4 * n + 1], from[4 * n + 2], from[4 * n + 3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (r0 + i < q.out_rows) {
                uint2 o;
                o.x = eight_bits(v[i][0], v[i][1], v[i][2], v[i][3], inverse);
                o.y = eight_bits(v[i][4], v[i][5], v[i][6], v[i][7], inverse);
                *(uint2 *)(out + (r0 + i) * kb * BLOCK8 + part * 8) = o;
            }
    }
}

bool rows_are_wide(const QuantArgs &q, int type)
{
    return ((uintptr_t)q.x & 15) == 0 && q.stride * (int64_t)type_size(type) % 16 == 0;
}

}  // namespace

hipError_t launch_quantize_rows(const QuantArgs &q, int type, hipStream_t s)
{
    const int64_t groups = q.out_rows * q.out_blocks, grid = (groups + 15) / 16;
    return with_type(type, [&](auto ty) {
        quantize_rows_kernel<decltype(ty)><<<(unsigned)(grid < (1 << 20) ? grid : (1 << 20)), 256, 0, s>>>(q, groups, rows_are_wide(q, type));
        return hipGetLastError();
    });
}

hipError_t launch_quantize_turned(const QuantArgs &q, int type, hipStream_t s)
{
    const int64_t strips = (q.cols + 63) / 64;
    const dim3 grid((unsigned)q.out_blocks, (unsigned)(strips < 1024 ? strips : 1024));
    return with_type(type, [&](auto ty) {
        quantize_turned_kernel<decltype(ty)><<<grid, 256, 0, s>>>(q, rows_are_wide(q, type));
        return hipGetLastError();
    });
}

hipError_t launch_quantize_both(const QuantArgs &q, const asgd_blocks &rows, int type, hipStream_t s)
{
    const int64_t strips = blocks8(q.cols);
    const dim3 grid((unsigned)q.out_blocks, (unsigned)(strips < 1024 ? strips : 1024));
    return with_type(type, [&](auto ty) {
        quantize_both_kernel<decltype(ty)><<<grid, 512, 0, s>>>(q, (uint8_t *)rows.values, rows.scales, rows.rows, blocks8(rows.cols), rows_are_wide(q, type));
        return hipGetLastError();
    });
}

hipError_t launch_quantize_squares(const QuantArgs &q, int type, bool turned, hipStream_t s)
{
    const int64_t squares = blocks8(q.out_rows) * q.out_blocks * q.count, across = squares < (1 << 16) ? squares : (1 << 16);
    const dim3 grid((unsigned)across, (unsigned)((squares + across - 1) / across));
    return with_type(type, [&](auto ty) {
        const bool wide = rows_are_wide(q, type);
        if (turned) quantize_squares_kernel<decltype(ty), true><<<grid, 256, 0, s>>>(q, wide);
        else quantize_squares_kernel<decltype(ty), false><<<grid, 256, 0, s>>>(q, wide);
        return hipGetLastError();
    });
}

}  // namespace asgd
