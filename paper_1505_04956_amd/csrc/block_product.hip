// Products of matrices in 8-bit blocks, out[m, n] = sum over blocks kb of sa[kb, m] sb[kb, n] sum over the block's 128 k of a[m, k] b[n, k], on the
// matrix cores (v_mfma_f32_16x16x128_f8f6f4: one instruction is one block of the contraction); sums and scales are 32-bit.  out^T = b a^T is what is formed: rows of b are the instruction's rows, rows of a its columns, so that a
// lane holds four neighbours of one row of out, and the scale of its row of a is one number a lane.
//
// The order of the 128 bytes of a block among the lanes is free as long as both operands have the same: lane l holds the
// sixteen bytes l / 16 and l / 16 + 4 of row l % 16.
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
__device__ __forceinline__ void to_lds4(const uint8_t *base, uint32_t offset, uint8_t *to)
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

// Many rows.  8192^3 to bfloat16: 453 us, 2.4 PFLOP/s, where the power that the card may draw holds its clock at 1.6 to 1.8 GHz (a
// library product with one scale for all reaches 2.65).  With 32-bit sums (EXACT) 8192^3 takes 898 us, 1.22 PFLOP/s; 65536 x 1024 x 128 to float32 is
// bound by memory, its 277 MB.  4096 rows of four of 64 experts, 2048 x 2048: 144 us, 0.95 PFLOP/s at 2.4 GHz, with 32-bit sums 182, 0.75;
// a wave waits for data of the LDS or of the other waves half of the time: a block begins with waits (below), experts' last tiles are part empty,
// and sixteen blocks are soon over.
//
// A tile of TOK rows of a and WT rows of b; the waves are TOK_WAVES x WT_WAVES, each with I x J pieces of 16 x 16.  Blocks of the
// contraction of both, and their scales, go straight to one of two or four (STAGES) stages in the LDS; 16-byte pieces of a row lie at their
// number xor the row's low bits, so that the lanes of a read spread over the banks.
//
// Within a block the rows of b are taken sixteen at a time: while the matrix cores work on one, the next is read from the
// LDS and the sums of earlier ones are scaled and added.  The one barrier of a block lies at its begin: by then its own loads have arrived and
// all waves are done with the block before, whose stage the block STAGES - 1 further on takes, loaded while the first of this one's rows
// are multiplied.  Nothing is read across the barrier, so a block's first rows of b, and its rows of a, are waited for.
template <int TOK, int WT, bool SQUARES> struct Stage {
    static constexpr int VALUES = (TOK + WT) * BLOCK8;                                      // bytes
    // pieces of 64 scales: the rows' of a; the rows' of b, or for squares one for 128 rows, 64 times over
    static constexpr int PIECES_A = (TOK + 63) / 64, PIECES_B = SQUARES ? (WT + BLOCK8 - 1) / BLOCK8 : (WT + 63) / 64, PIECES = PIECES_A + PIECES_B;
    static constexpr int SCALES_B = VALUES + PIECES_A * 256, BYTES = VALUES + PIECES * 256;
};

template <int TOK, int WT, int TOK_WAVES, int WT_WAVES, int STAGES, bool SQUARES, bool EXACT, bool FAR, class Out>
__global__ __launch_bounds__(64 * TOK_WAVES * WT_WAVES, 2) void product_kernel(ProductArgs p, uint32_t tiles_tok, uint32_t tiles_wt, bool wide)
{
    typedef Stage<TOK, WT, SQUARES> S;
    constexpr int WAVES = TOK_WAVES * WT_WAVES, J = TOK / TOK_WAVES / 16, I = WT / WT_WAVES / 16;
    constexpr int SEGMENTS = (TOK + WT) / 8 / WAVES;             // of eight rows, that a wave brings
    constexpr int PIECES = (S::PIECES + WAVES - 1) / WAVES;      // of 64 scales
    static_assert((TOK + WT) / 8 % WAVES == 0 && WT / WT_WAVES <= BLOCK8 && TOK % (16 * TOK_WAVES) == 0 && WT % (16 * WT_WAVES) == 0, "");
    __shared__ __align__(16) uint8_t stage0[S::BYTES];
    __shared__ __align__(16) uint8_t stage1[S::BYTES];
    __shared__ __align__(16) uint8_t stage2[STAGES > 2 ? S::BYTES : 16];
    __shared__ __align__(16) uint8_t stage3[STAGES > 3 ? S::BYTES : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_tok = wave % TOK_WAVES * (J * 16), wave_wt = wave / TOK_WAVES * (I * 16);

    // which tile: strips of eight tiles of a, all tiles of b for each.  (The host knows how many tiles experts can have at most; shared among
    // the dies are those that they have.)
    const bool grouped = SQUARES && TOK == BLOCK8 && (p.mode == ASGD_PRODUCT_GATHER || p.mode == ASGD_PRODUCT_PLACES);
    const bool over = !SQUARES && TOK == BLOCK8 && p.mode == ASGD_PRODUCT_OVER;
    if (grouped) tiles_tok = p.order.blocks[p.order.E];
    const uint32_t all = grouped ? tiles_tok * tiles_wt : gridDim.x;
    if (blockIdx.x >= all) return;
    const uint32_t id = tile_of_group(blockIdx.x, all);
    uint32_t within = id;
    int64_t matrix = 0;
    if (over) {
        matrix = id / (tiles_tok * tiles_wt);
        within = id - (uint32_t)matrix * tiles_tok * tiles_wt;
    }
    const uint32_t strip = within / (8 * tiles_wt), in_strip = within - strip * 8 * tiles_wt;
    const uint32_t high = min(tiles_tok - strip * 8, 8u), tile_wt = in_strip / high, tile_tok = strip * 8 + in_strip - tile_wt * high;

    int64_t first = (int64_t)tile_tok * TOK, end = p.rows_a;
    int k0 = 0, k1 = (int)p.kb;
    const int64_t first_wt = (int64_t)tile_wt * WT;
    if (grouped) {
        int e;
        if (!block_of_expert(p.order, tile_tok, e, first, end)) return;
        matrix = e;
    } else if (over) {
        k0 = p.order.blocks[matrix];
        k1 = p.order.blocks[matrix + 1];
    }
    const int64_t row_bytes = p.kb * BLOCK8, b_matrix = over ? 0 : matrix * p.rows_b;
    const auto row_of_a = [&](int64_t r) {                        // (rows beyond the last: the last again)
        r = r < end ? r : end - 1;
        return grouped && p.mode == ASGD_PRODUCT_GATHER ? (int64_t)(p.order.slots[r] / p.order.k) : r;
    };
    const auto row_of_b = [&](int64_t r) { return r < p.rows_b ? r : p.rows_b - 1; };

    // Where a lane's pieces come from, in bytes from the tile's first row.  Neighbouring rows of a tile are less than 2^32 bytes apart;
    // gathered ones may be further (FAR)
    typedef typename std::conditional<FAR, uint64_t, uint32_t>::type Offset;
    Offset from[SEGMENTS];
    const int64_t first_a = row_of_a(first);
    const uint8_t *const a_base = p.a + first_a * row_bytes, *const b_base = p.b + (b_matrix + first_wt) * row_bytes;
#pragma unroll
    for (int s = 0; s < SEGMENTS; s++) {
        const int row = (wave * SEGMENTS + s) * 8 + (lane >> 3), piece = (lane & 7) ^ (lane >> 3);
        const int64_t r = row < TOK ? row_of_a(first + row) - first_a : row_of_b(first_wt + row - TOK) - first_wt;
        from[s] = (Offset)(r * row_bytes + piece * 16);
    }
    // and its scales: a run of 64 rows, or (squares) one number for all lanes
    uint32_t scale_row[PIECES];                                  // bytes
    const float *scale_from[PIECES];
    int64_t scale_step[PIECES];                                  // from block to block
#pragma unroll
    for (int s = 0; s < PIECES; s++) {
        const int piece = (wave + s * WAVES) % S::PIECES;         // (some twice: the same numbers to the same places)
        const int64_t at = first_wt / BLOCK8 + (piece - S::PIECES_A), nb = blocks8(p.rows_b);
        const bool of_a = piece < S::PIECES_A;
        scale_row[s] = 4 * (uint32_t)(of_a ? row_of_a(first + piece * 64 + lane) : SQUARES ? 0 : row_of_b(first_wt + (piece - S::PIECES_A) * 64 + lane));
        scale_from[s] = of_a ? p.sa : SQUARES ? p.sb + (matrix * nb + (at < nb ? at : nb - 1)) * p.kb : p.sb;
        scale_step[s] = of_a ? p.rows_a : SQUARES ? 1 : p.rows_b;
    }
    constexpr int LOADS = SEGMENTS + PIECES, LOADING = I > 1 ? 2 : 1;  // of a wave for a block; over so many of its steps
    const auto bring = [&](int kb, uint8_t *stage, int l) {      // the l-th of a wave's loads of a block
        if (l < SEGMENTS) {
            const int segment = wave * SEGMENTS + l;
            asm volatile("" : "+v"(from[l]));                     // (else its sum with the base is kept, in twice the registers)
            to_lds((segment * 8 < TOK ? a_base : b_base) + (int64_t)kb * BLOCK8, from[l], stage + segment * 1024);
        } else {
            const int s = l - SEGMENTS;
            asm volatile("" : "+v"(scale_row[s]));
            to_lds4((const uint8_t *)(scale_from[s] + kb * scale_step[s]), scale_row[s], stage + S::VALUES + (wave + s * WAVES) % S::PIECES * 256);
        }
    };

    v4f sum[I][J];
#pragma unroll
    for (int i = 0; i < I; i++)
#pragma unroll
        for (int j = 0; j < J; j++) sum[i][j] = {0.0f, 0.0f, 0.0f, 0.0f};

    // A lane's places in a stage: its pieces of the first sixteen rows of each operand, its scales.  (Opaque, so that all reads are a
    // register and a constant.)
    const int low = ((lane >> 4) ^ (lane & 7)) * 16;
    int at_a = (wave_tok + (lane & 15)) * BLOCK8 + low, at_w = (TOK + wave_wt + (lane & 15)) * BLOCK8 + low;
    int at_sa = S::VALUES + (wave_tok + (lane & 15)) * 4, at_sb = S::SCALES_B + (SQUARES ? wave_wt / BLOCK8 * 256 + lane * 4 : wave_wt * 4 + (lane >> 4) * 16);
    asm volatile("" : "+v"(at_a), "+v"(at_w), "+v"(at_sa), "+v"(at_sb));
    struct Raw { v4i u, v; };
    const auto operand = [&](const uint8_t *stage, int at, int rows) {
        return Raw{*(const v4i *)(stage + at + rows * BLOCK8), *(const v4i *)(stage + (at ^ 64) + rows * BLOCK8)};
    };
    // multiplies the block in `stage` and brings block `next` to `other`
    const auto multiply = [&](const uint8_t *stage, int next, uint8_t *other, auto bringing) {
        constexpr bool BRING = decltype(bringing)::value;
        constexpr int LAG = 2, N = I * J, PER = (LOADS + LOADING - 1) / LOADING;
        float s[J];
        Operand<EXACT> a[J], w;
        Raw raw[J], after = operand(stage, at_w, 0);              // (converted where it is used: not to wait for it where it is read)
        v4f part[LAG + 1], sb[2];
#pragma unroll
        for (int j = 0; j < J; j++) {
            raw[j] = operand(stage, at_a, j * 16);
            s[j] = *(const float *)(stage + at_sa + j * 64);
        }
#pragma unroll
        for (int j = 0; j < J; j++) a[j].set(raw[j].u, raw[j].v);
        if (SQUARES) {
            const float of_b = *(const float *)(stage + at_sb);
#pragma unroll
            for (int j = 0; j < J; j++) s[j] *= of_b;
        }
        const auto row = [&](int i) {                             // begins sixteen rows of b
            w.set(after.u, after.v);
            if (i + 1 < I) after = operand(stage, at_w, (i + 1) * 16);
            if (!SQUARES) sb[i & 1] = *(const v4f *)(stage + at_sb + i * 64);
            if (BRING && i < LOADING)
#pragma unroll
                for (int l = i * PER; l < (i + 1) * PER && l < LOADS; l++) bring(next, other, l);
        };
        if constexpr (EXACT) {
            // a quarter of a block for all J, then the next: each instruction adds to what the one J before it gives; one sum of the rows before beside each
            v4f parts[2][J];
#pragma unroll
            for (int q = 0; q < (I + 1) * 4 * J; q++) {
                const int i = q / (4 * J), n = q / J % 4, j = q % J;
                if (i < I) {
                    if (q % (4 * J) == 0) row(i);
                    const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
                    parts[i & 1][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[n], a[j].v[n], n == 0 ? zero : parts[i & 1][j], 0, 0, 0);
                }
                if (i > 0) {
                    const float got = parts[(i - 1) & 1][j][n];
                    sum[i - 1][j][n] = fmaf(SQUARES ? got : got * sb[(i - 1) & 1][n], s[j], sum[i - 1][j][n]);
                    if (n == 3) asm volatile("" : "+v"(sum[i - 1][j]));     // (here, and not after the next barrier)
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int q = 0; q < N + LAG; q++) {
                if (q < N) {
                    if (q % J == 0) row(q / J);
                    part[q % (LAG + 1)] = block_product(w, a[q % J]);
                }
                if (q >= LAG) {
                    const int i = (q - LAG) / J, j = (q - LAG) % J;
                    const v4f got = part[(q - LAG) % (LAG + 1)];
#pragma unroll
                    for (int n = 0; n < 4; n++) sum[i][j][n] = fmaf(SQUARES ? got[n] : got[n] * sb[i & 1][n], s[j], sum[i][j][n]);
                    asm volatile("" : "+v"(sum[i][j]));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };

    // Step n of a round multiplies stage n and fills the one that was multiplied before it with the block STAGES - 1 further on (the last
    // block once more where there is none left).  Before that a wave's loads of this block have arrived, those of later ones need not have,
    // and all waves are done with the stage that is filled.
    const auto step = [&](int kb, auto at) {
        constexpr int N = decltype(at)::value % STAGES, FREE = (N + STAGES - 1) % STAGES;
        uint8_t *const stages[4] = {stage0, stage1, stage2, stage3};
        constexpr int FLYING = (STAGES - 2) * LOADS;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((FLYING & 15) | 7 << 4 | 15 << 8 | FLYING >> 4 << 14);       // (vmcnt alone)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        multiply(stages[N], min(kb + STAGES - 1, k1 - 1), stages[FREE], std::true_type());
    };
    if (k0 < k1) {
        uint8_t *const stages[4] = {stage0, stage1, stage2, stage3};
#pragma unroll
        for (int n = 0; n < STAGES - 1; n++)
#pragma unroll
            for (int l = 0; l < LOADS; l++) bring(min(k0 + n, k1 - 1), stages[n], l);
        int kb = k0;
        for (; kb + STAGES - 1 < k1; kb += STAGES) {
            step(kb, One<0>());
            step(kb + 1, One<1>());
            if constexpr (STAGES > 2) step(kb + 2, One<2>());
            if constexpr (STAGES > 3) step(kb + 3, One<3>());
        }
        if (kb < k1) step(kb, One<0>());
        if constexpr (STAGES > 2)
            if (kb + 1 < k1) step(kb + 1, One<1>());
        if constexpr (STAGES > 3)
            if (kb + 2 < k1) step(kb + 2, One<2>());
    }

    // Out through the LDS, sixteen rows of a at a time: there a lane has four neighbours of a row, in memory whole lines are wanted.
    typedef typename Out::T T;
    constexpr int ROW = I * 16 * sizeof(T), PITCH = ROW + 16, PER_ROW = ROW / 16, ROWS = 64 / PER_ROW;       // bytes; lanes of a row, rows of an instruction
    T *out = (T *)p.out + (over ? matrix * p.rows_a * p.stride : 0);
    // (the last steps brought the last block once more: to stages that results go to now, so it has to be there before any wave's barrier)
    __builtin_amdgcn_s_waitcnt(7 << 4 | 15 << 8);                 // (vmcnt alone, to zero)
    __syncthreads();
    constexpr int HALF = (WAVES + 1) / 2;
    static_assert(HALF * 16 * PITCH <= S::BYTES, "");
    uint8_t *mine = (wave < HALF ? stage0 : stage1) + (wave < HALF ? wave : wave - HALF) * 16 * PITCH;
#pragma unroll
    for (int j = 0; j < J; j++) {
#pragma unroll
        for (int i = 0; i < I; i++) {
            T u[4] = {(T)sum[i][j][0], (T)sum[i][j][1], (T)sum[i][j][2], (T)sum[i][j][3]};
            uint8_t *to = mine + (lane & 15) * PITCH + (i * 16 + (lane >> 4) * 4) * sizeof(T);
            if constexpr (sizeof(T) == 4) *(uint4 *)to = *(uint4 *)u;
            else *(uint2 *)to = *(uint2 *)u;
        }
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
#pragma unroll
        for (int n = 0; n < 16 / ROWS; n++) {
            const int row = n * ROWS + lane / PER_ROW, at = lane % PER_ROW * 16;
            const int64_t r = first + wave_tok + j * 16 + row, c = first_wt + wave_wt + at / sizeof(T);
            const v4i v = *(const v4i *)(mine + row * PITCH + at);
            if (r < end) store16<T>(out + r * p.stride + c, p.rows_b - c, wide, v);
        }
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
    }
}

// ---- few rows ---------------------------------------------------------------------------------------------------------
// What counts is that the weights arrive: they go from memory to registers, sixteen rows of one block of 128 a wave and
// instruction, and the eight waves of a workgroup share the blocks of the contraction of sixteen rows of b, four of them on
// their way at a time.  Rows of a, J times sixteen, come from the caches; RAW ones are brought to 8 bits in the registers of
// the lanes that need them (up to sixteen of them: there this is less than a launch costs).  One row times 4096 x 4096: 9.0 us, 1.9
// TB/s; 120 rows of 100 experts, 33 of which have rows, 1000 x 1100: 18 us, 2.1 TB/s.  The weights' way from memory bounds it, one round of loads a wave at few strips.
constexpr int FEW_WAVES = 8;

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

// In: void, or the type of a RAW a (J = 1).  A workgroup takes STRIPS times sixteen rows of b, whose loads of a block are on their way
// together, or (one strip) those of four blocks.  grid: groups of strips, tiles of a
template <class In, int J, int STRIPS, bool SQUARES, bool EXACT, class Out> __global__ __launch_bounds__(64 * FEW_WAVES) void product_few_kernel(ProductArgs p, bool wide_in, bool wide)
{
    constexpr bool RAW = !std::is_same<In, void>::value;
    constexpr int AHEAD = STRIPS == 1 ? 4 : 1;
    __shared__ v4f parts[FEW_WAVES][J * STRIPS][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t strip = (int64_t)blockIdx.x * STRIPS;
    int64_t matrix = 0, first = (int64_t)blockIdx.y * (16 * J), end = p.rows_a;
    if (p.mode == ASGD_PRODUCT_GATHER || p.mode == ASGD_PRODUCT_PLACES) {
        int e;
        if (!tile_of_expert(p.order, blockIdx.y, 16 * J, e, first, end)) return;
        matrix = e;
    }
    const int tok = lane & 15, quarter = lane >> 4;
    int64_t src[J];
#pragma unroll
    for (int j = 0; j < J; j++) {
        const int64_t r = first + j * 16 + tok < end ? first + j * 16 + tok : end - 1;       // (rows beyond the last: the last again)
        src[j] = p.mode == ASGD_PRODUCT_GATHER ? p.order.slots[r] / p.order.k : r;
    }
    const int64_t row_bytes = p.kb * BLOCK8, squares = blocks8(p.rows_b);
    const uint8_t *b[STRIPS];
#pragma unroll
    for (int s = 0; s < STRIPS; s++) {
        const int64_t r = (strip + s) * 16 + tok;
        b[s] = p.b + (matrix * p.rows_b + (r < p.rows_b ? r : p.rows_b - 1)) * row_bytes + quarter * 32;
    }
    v4f sum[STRIPS][J];
#pragma unroll
    for (int s = 0; s < STRIPS; s++)
#pragma unroll
        for (int j = 0; j < J; j++) sum[s][j] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t kb0 = wave; kb0 < p.kb; kb0 += FEW_WAVES * AHEAD) {
        v4i u[STRIPS][AHEAD], v[STRIPS][AHEAD];
        RawBlock<In> raw[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; n++) {
            const int64_t kb = kb0 + n * FEW_WAVES < p.kb ? kb0 + n * FEW_WAVES : kb0;
            if constexpr (RAW) raw[n].load((const typename In::T *)p.a + src[0] * p.stride_raw, first + tok < end, wide_in, kb * BLOCK8 + quarter * 32, p.cols);
#pragma unroll
            for (int s = 0; s < STRIPS; s++) {
                u[s][n] = *(const v4i *)(b[s] + kb * BLOCK8);
                v[s][n] = *(const v4i *)(b[s] + kb * BLOCK8 + 16);
            }
        }
#pragma unroll
        for (int n = 0; n < AHEAD; n++) {
            // Past the last block: the first of these again, times zero.  (Not a branch around the sums: a matrix instruction whose result a path
            // leaves unused writes registers that the path has taken for something else by then, addresses among them.)
            const bool there = kb0 + n * FEW_WAVES < p.kb;
            const int64_t kb = there ? kb0 + n * FEW_WAVES : kb0;
            Operand<EXACT> a[J];
            float scale[J];
#pragma unroll
            for (int j = 0; j < J; j++) {
                v4i lo, hi;
                if constexpr (RAW) raw[n].set(first + tok < end, scale[j], lo, hi);
                else {
                    const uint8_t *at = p.a + src[j] * row_bytes + kb * BLOCK8 + quarter * 32;
                    lo = *(const v4i *)at;
                    hi = *(const v4i *)(at + 16);
                    scale[j] = p.sa[kb * p.rows_a + src[j]];
                }
                a[j].set(lo, hi);
                scale[j] = there ? scale[j] : 0.0f;
            }
#pragma unroll
            for (int s = 0; s < STRIPS; s++) {
                Operand<EXACT> w;
                w.set(u[s][n], v[s][n]);
                v4f of_b;
                const int64_t row = (strip + s) * 16;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    if (SQUARES) of_b[i] = p.sb[(matrix * squares + (row / BLOCK8 < squares ? row / BLOCK8 : squares - 1)) * p.kb + kb];
                    else of_b[i] = p.sb[kb * p.rows_b + (row + quarter * 4 + i < p.rows_b ? row + quarter * 4 + i : p.rows_b - 1)];
                }
#pragma unroll
                for (int j = 0; j < J; j++) {
                    const v4f part = block_product(w, a[j]);
#pragma unroll
                    for (int i = 0; i < 4; i++) sum[s][j][i] = SQUARES ? fmaf(part[i], scale[j] * of_b[i], sum[s][j][i]) : fmaf(part[i] * of_b[i], scale[j], sum[s][j][i]);
                }
            }
        }
    }
#pragma unroll
    for (int s = 0; s < STRIPS; s++)
#pragma unroll
        for (int j = 0; j < J; j++) parts[wave][s * J + j][lane] = sum[s][j];
    __syncthreads();
    for (int n = wave; n < J * STRIPS; n += FEW_WAVES) {
        v4f total = parts[0][n][lane];
#pragma unroll
        for (int w = 1; w < FEW_WAVES; w++) total += parts[w][n][lane];
        const int64_t row = first + n % J * 16 + tok, c = (strip + n / J) * 16 + quarter * 4;
        if (row < end) store_four<Out>((typename Out::T *)p.out + row * p.stride + c, p.rows_b - c, wide, total);
    }
}

// A row's experts without an order, for few rows: a workgroup takes sixteen rows of b of every expert of one row of a (blockIdx.y), and
// adds what they give times its weights.  A block of the row is brought to 8 bits once for all of them; the weights of up to
// EXPERTS of them are on their way at a time.  Six experts of 2048 x 2048: 10.0 us, 2.5 TB/s.  Sixteen waves, since a round of loads then
// is all that each has of 2048 columns, and its latency is what counts (eight: 10.4).
constexpr int DIRECT_WAVES = 16;

template <class In, bool EXACT, class Out> __global__ __launch_bounds__(64 * DIRECT_WAVES) void product_direct_kernel(ProductArgs p, const int32_t *ids, const float *weights, int k, int E, bool wide_in, bool wide)
{
    constexpr int EXPERTS = 4;
    __shared__ v4f parts[DIRECT_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tok = lane & 15, quarter = lane >> 4;
    const int64_t t = blockIdx.y, strip = blockIdx.x, r = strip * 16 + tok, row_bytes = p.kb * BLOCK8;
    const uint8_t *b = p.b + (r < p.rows_b ? r : p.rows_b - 1) * row_bytes + quarter * 32;
    const float *sb = p.sb + strip / 8 * p.kb;
    const int64_t matrix = p.rows_b * row_bytes, squares = blocks8(p.rows_b) * p.kb;
    const typename In::T *row = (const typename In::T *)p.a + t * p.stride_raw;
    v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t kb = wave; kb < p.kb; kb += DIRECT_WAVES) {
        float scale;
        v4i lo, hi;
        Operand<EXACT> a;
        RawBlock<In> raw;
        raw.load(row, tok == 0, wide_in, kb * BLOCK8 + quarter * 32, p.cols);
        for (int j0 = 0; j0 < k; j0 += EXPERTS) {
            v4i u[EXPERTS], v[EXPERTS];
            float of_b[EXPERTS];
#pragma unroll
            for (int j = 0; j < EXPERTS; j++) {
                const int e = j0 + j < k ? ids[t * k + j0 + j] : -1;
                const bool there = (unsigned)e < (unsigned)E;
                const int64_t m = there ? e : 0;
                of_b[j] = there ? sb[m * squares + kb] * weights[t * k + j0 + j] : 0.0f;
                if (there) {
                    u[j] = *(const v4i *)(b + m * matrix + kb * BLOCK8);
                    v[j] = *(const v4i *)(b + m * matrix + kb * BLOCK8 + 16);
                }
            }
            if (j0 == 0) {
                raw.set(tok == 0, scale, lo, hi);
                a.set(lo, hi);
            }
#pragma unroll
            for (int j = 0; j < EXPERTS; j++) {
                const int e = j0 + j < k ? ids[t * k + j0 + j] : -1;
                if ((unsigned)e < (unsigned)E) {
                    Operand<EXACT> w;
                    w.set(u[j], v[j]);
                    const v4f part = block_product(w, a);
#pragma unroll
                    for (int i = 0; i < 4; i++) sum[i] = fmaf(part[i], scale * of_b[j], sum[i]);
                }
            }
        }
    }
    parts[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && tok == 0) {
#pragma unroll
        for (int w = 1; w < DIRECT_WAVES; w++) sum += parts[w][lane];
        const int64_t c = strip * 16 + quarter * 4;
        store_four<Out>((typename Out::T *)p.out + t * p.stride + c, p.rows_b - c, wide, sum);
    }
}

}  // namespace

// places in use by `slots` slots of E experts, each expert's rounded up to whole tiles: what there can be at most, and what there will be about
static int64_t most_tiles(int64_t slots, int64_t E, int rows) { return slots / rows + (slots < E ? slots : E); }

// Which tile: us of a block of the contraction for n tiles on 256 compute units, from what one tile takes with a unit to itself and what each takes where
// there are many, the writing of results included (8-bit instruction, squares): 64 x 64 0.31 and 0.223, 128 x 128 0.66 and 0.63, 256 x 256 2.1.  What
// each takes, and so what the rule decides between, in that order: 777 x 1001 x 1152 7.2, 11.4, 29.4 us; 256 x 4096 x 4096 11.1, 21.6, 46.4; 2048^3
// 17.6, 14.7, 28.0; 4096 x 4096 x 2048 67, 46.5, 41.4; 8192^3 821, 542, 453.  Sums in 32 bits take about twice as long in each, and have no
// 256 x 256 (registers).
static double tiles_time(int64_t n, double alone, double among) { return n <= 256 ? alone : alone > (double)((n + 255) / 256) * among ? alone : (double)((n + 255) / 256) * among; }

// Four strips a workgroup (its rows of a, its place among the experts and its end are then there once for four) where that leaves more than a workgroup for
// each of the 256 compute units, or the contraction has less than a block for each of its waves.
static bool more_strips(const ProductArgs &p, unsigned strips, unsigned tiles) { return (int64_t)strips * tiles >= 2048 || (p.kb <= FEW_WAVES && strips >= 4); }

static bool experts_rows(const ProductArgs &p) { return p.mode == ASGD_PRODUCT_GATHER || p.mode == ASGD_PRODUCT_PLACES; }

// rows of a (of an expert, on average)
static int64_t rows_each(const ProductArgs &p) { return experts_rows(p) ? p.order.T * p.order.k / p.order.E : p.rows_a; }

int product_form(const ProductArgs &p, bool squares)
{
    const bool over = p.mode == ASGD_PRODUCT_OVER;
    if (!over && rows_each(p) <= 32) return ASGD_PRODUCT_FORM_FEW;
    if (experts_rows(p)) return (double)p.rows_a * p.kb * BLOCK8 >= 4294967296.0 ? ASGD_PRODUCT_FORM_TILES_128_FAR : ASGD_PRODUCT_FORM_TILES_128;
    if (over) return ASGD_PRODUCT_FORM_TILES_128;
    const auto tiles = [&](int n) { return ((p.rows_a + n - 1) / n) * ((p.rows_b + n - 1) / n); };
    const double t64 = tiles_time(tiles(64), 0.31, 0.223), t128 = tiles_time(tiles(128), 0.66, 0.63);
    if (t64 < t128) return ASGD_PRODUCT_FORM_TILES_64;
    return squares && !p.exact && tiles_time(tiles(256), 2.1, 2.1) < t128 ? ASGD_PRODUCT_FORM_TILES_256 : ASGD_PRODUCT_FORM_TILES_128;
}

hipError_t launch_product(const ProductArgs &p, bool squares, int type, hipStream_t s)
{
    const bool grouped = experts_rows(p), over = p.mode == ASGD_PRODUCT_OVER;
    const int64_t slots = grouped ? p.order.T * p.order.k : 0, E = p.order.E;
    const int form = product_form(p, squares);
    const bool wide4 = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * type_size(type)) == 0;
    const bool wide16 = p.stride * type_size(type) % 16 == 0 && (uintptr_t)p.out % 16 == 0;
    const auto tiles_of = [&](int tok) { return grouped ? most_tiles(slots, E, tok) : (p.rows_a + tok - 1) / tok; };
    return with_type(type, [&](auto out) {
        typedef decltype(out) Out;
        const auto few = [&](auto j, auto sq, auto exact) {
            constexpr int J = decltype(j)::value;
            const unsigned strips = (unsigned)((p.rows_b + 15) / 16), tiles = (unsigned)tiles_of(16 * J);
            if (!more_strips(p, strips, tiles)) product_few_kernel<void, J, 1, decltype(sq)::value, decltype(exact)::value, Out><<<dim3(strips, tiles), 64 * FEW_WAVES, 0, s>>>(p, false, wide4);
            else product_few_kernel<void, J, 4, decltype(sq)::value, decltype(exact)::value, Out><<<dim3((strips + 3) / 4, tiles), 64 * FEW_WAVES, 0, s>>>(p, false, wide4);
            return hipGetLastError();
        };
        const auto tiles = [&](auto tok, auto wt, auto waves_tok, auto waves_wt, auto stages, auto sq, auto exact, auto far) {
            constexpr int TOK = decltype(tok)::value, WT = decltype(wt)::value, WAVES = decltype(waves_tok)::value * decltype(waves_wt)::value;
            const int64_t tiles_tok = tiles_of(TOK), tiles_wt = (p.rows_b + WT - 1) / WT;
            product_kernel<TOK, WT, decltype(waves_tok)::value, decltype(waves_wt)::value, decltype(stages)::value, decltype(sq)::value, decltype(exact)::value, decltype(far)::value, Out>
                <<<(unsigned)(tiles_tok * tiles_wt * (over ? E : 1)), 64 * WAVES, 0, s>>>(p, (uint32_t)tiles_tok, (uint32_t)tiles_wt, wide16);
            return hipGetLastError();
        };
        const auto choose = [&](auto sq, auto exact) {
            const std::true_type yes;
            const std::false_type no;
            if (form == ASGD_PRODUCT_FORM_FEW) return rows_each(p) <= 16 ? few(One<1>(), sq, exact) : few(One<2>(), sq, exact);
            if constexpr (decltype(sq)::value)                    // (experts' weights are squares)
                if (form == ASGD_PRODUCT_FORM_TILES_128_FAR) return tiles(One<128>(), One<128>(), One<2>(), One<2>(), One<2>(), sq, exact, yes);
            if (form == ASGD_PRODUCT_FORM_TILES_64) return tiles(One<64>(), One<64>(), One<2>(), One<2>(), One<4>(), sq, exact, no);
            if constexpr (!decltype(exact)::value && decltype(sq)::value)
                if (form == ASGD_PRODUCT_FORM_TILES_256) return tiles(One<256>(), One<256>(), One<4>(), One<2>(), One<2>(), sq, exact, no);
            return tiles(One<128>(), One<128>(), One<2>(), One<2>(), One<2>(), sq, exact, no);
        };
        const std::true_type yes;
        const std::false_type no;
        return squares ? p.exact ? choose(yes, yes) : choose(yes, no) : p.exact ? choose(no, yes) : choose(no, no);
    });
}

hipError_t launch_product_direct(const ProductArgs &p, const int32_t *ids, const float *weights, int k, int E, int raw_type, int type, hipStream_t s)
{
    const bool wide = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * type_size(type)) == 0;
    const bool wide_in = p.stride_raw * (int64_t)type_size(raw_type) % 16 == 0 && ((uintptr_t)p.a & 15) == 0;
    const dim3 grid((unsigned)((p.rows_b + 15) / 16), (unsigned)p.rows_a);
    return with_type(raw_type, [&](auto in) {
        return with_type(type, [&](auto out) {
            if (p.exact) product_direct_kernel<decltype(in), true, decltype(out)><<<grid, 64 * DIRECT_WAVES, 0, s>>>(p, ids, weights, k, E, wide_in, wide);
            else product_direct_kernel<decltype(in), false, decltype(out)><<<grid, 64 * DIRECT_WAVES, 0, s>>>(p, ids, weights, k, E, wide_in, wide);
            return hipGetLastError();
        });
    });
}

hipError_t launch_product_raw(const ProductArgs &p, int raw_type, int type, hipStream_t s)
{
    const bool grouped = p.mode == ASGD_PRODUCT_GATHER;
    const bool wide = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * type_size(type)) == 0;
    const bool wide_in = p.stride_raw * (int64_t)type_size(raw_type) % 16 == 0 && ((uintptr_t)p.a & 15) == 0;
    const unsigned strips = (unsigned)((p.rows_b + 15) / 16), tiles = grouped ? (unsigned)most_tiles(p.order.T * p.order.k, p.order.E, 16) : 1u;
    const bool more = more_strips(p, strips, tiles);
    const dim3 grid(more ? (strips + 3) / 4 : strips, tiles);
    return with_type(raw_type, [&](auto in) {
        return with_type(type, [&](auto out) {
            const auto go = [&](auto n, auto exact) {
                product_few_kernel<decltype(in), 1, decltype(n)::value, true, decltype(exact)::value, decltype(out)><<<grid, 64 * FEW_WAVES, 0, s>>>(p, wide_in, wide);
                return hipGetLastError();
            };
            const std::true_type yes;
            const std::false_type no;
            return more ? p.exact ? go(One<4>(), yes) : go(One<4>(), no) : p.exact ? go(One<1>(), yes) : go(One<1>(), no);
        });
    });
}

}  // namespace asgd
