// Products of matrices in 4 bits, out[m, n] = sum over blocks of 32 of sa sb sum over the block's k of a[m, k] b[n, k], on the matrix cores
// (v_mfma_f32_16x16x128_f8f6f4 with both operands e2m1): one instruction takes four blocks of 16 rows of each operand, their scales among its
// operands, and adds to 32-bit sums.  What it adds is exact to 1.2e-7 of the products' magnitudes (measured; products of e2m1 numbers are multiples of
// 1/4 up to 36, so that nothing of them is dropped where eight of them are aligned).  As in 8 bits rows of b are the instruction's rows, and a lane
// holds four neighbours of one row of out.
#include "four_bits.h"

namespace asgd {

namespace {

// ---- many rows ----------------------------------------------------------------------------------------------------
// A tile of TOK rows of a and WT rows of b; the waves are TOK_WAVES x WT_WAVES, each with I x J pieces of 16 x 16.  A stage in the LDS is a run of 256
// columns of all rows, 128 bytes of values each, filled straight from memory while others are multiplied; sixteen-byte pieces of a row lie at their number xor the
// row's low bits, so that the lanes of a read spread over the banks.  A row's scales are eight bytes of a run: they come for four runs at a time, 32 bytes of a
// row, since what counts for memory is how many lines are asked for (a run at a time they were as many as the values'), to one of two places of
// their own, eight bytes of a row at their number xor two of the row's bits.
//
// 8192^3 to bfloat16: 259 to 282 us, 3.9 to 4.2 PFLOP/s (a library product with the same scales: 3.6; scales a run at a time: 296); with one of 64 products of a run left
// it takes 203, without the results 265.  4093 rows of four of 64 experts, 2048 x 2048, to float32: 89 us (scales a run at a time: 103), with one of 32 products left 91,
// without the results 74, with one run of the eight 32, without either 25: the operands' way from the second caches to the LDS bounds it, 0.7 GB in the 49 us of
// seven runs, and what a tile begins with (its expert, its rows, its first loads).  Eight waves of 64 x 32 took 103 where four of 64 x 64 took 111, two workgroups of two
// stages a compute unit 111 where one of four took 134, tiles of 128 x 256 99 where 128 x 128 take 89.
template <int TOK, int WT, int TOK_WAVES, int WT_WAVES, int STAGES, bool GROUPED, class Out>
__global__ __launch_bounds__(64 * TOK_WAVES * WT_WAVES, 2) void product_four_kernel(ProductArgs p, uint32_t tiles_tok, uint32_t tiles_wt, bool wide)
{
    constexpr int WAVES = TOK_WAVES * WT_WAVES, J = TOK / TOK_WAVES / 16, I = WT / WT_WAVES / 16, ROWS_ALL = TOK + WT, ROUND = 4;
    constexpr int SEGMENTS = ROWS_ALL / 8 / WAVES;               // of eight rows, that a wave brings: values of a run, and scales of four
    constexpr int BYTES = ROWS_ALL * RUN4_BYTES, SCALES = ROWS_ALL * RUN4_SCALES * ROUND;
    static_assert(ROWS_ALL / 8 % WAVES == 0 && SEGMENTS % 2 == 0 && TOK % (16 * TOK_WAVES) == 0 && WT % (16 * WT_WAVES) == 0 && (STAGES == 2 || STAGES == 4), "");
    __shared__ __align__(16) uint8_t stage0[BYTES];
    __shared__ __align__(16) uint8_t stage1[BYTES];
    __shared__ __align__(16) uint8_t stage2[STAGES > 2 ? BYTES : 16];
    __shared__ __align__(16) uint8_t stage3[STAGES > 3 ? BYTES : 16];
    __shared__ __align__(16) uint8_t scales[2][SCALES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_tok = wave % TOK_WAVES * (J * 16), wave_wt = wave / TOK_WAVES * (I * 16);

    // which tile: strips of eight tiles of a, all tiles of b for each
    if (GROUPED) tiles_tok = p.order.blocks[p.order.E];
    const uint32_t all = GROUPED ? tiles_tok * tiles_wt : gridDim.x;
    if (blockIdx.x >= all) return;
    const uint32_t id = tile_of_group(blockIdx.x, all);
    const uint32_t strip = id / (8 * tiles_wt), in_strip = id - strip * 8 * tiles_wt;
    const uint32_t high = min(tiles_tok - strip * 8, 8u), tile_wt = in_strip / high, tile_tok = strip * 8 + in_strip - tile_wt * high;

    int64_t first = (int64_t)tile_tok * TOK, end = p.rows_a, matrix = 0;
    const int64_t first_wt = (int64_t)tile_wt * WT;
    if (GROUPED) {
        static_assert(!GROUPED || TOK == BLOCK8, "");
        int e;
        if (!block_of_expert(p.order, tile_tok, e, first, end)) return;
        matrix = e;
    }
    const int64_t row_bytes = p.kb * RUN4_BYTES, scale_bytes = p.kb * RUN4_SCALES;
    const auto row_of_a = [&](int64_t r) {                        // (rows beyond the last: the last again)
        r = r < end ? r : end - 1;
        return GROUPED && p.mode == ASGD_PRODUCT_GATHER ? (int64_t)(p.order.slots[r] / p.order.k) : r;
    };
    const auto row_of_b = [&](int64_t r) { return r < p.rows_b ? r : p.rows_b - 1; };

    // Where a lane's pieces come from, in bytes from the tile's first row (gathered rows of a may be further apart than 2^32)
    typedef typename std::conditional<GROUPED, uint64_t, uint32_t>::type Offset;
    Offset from[SEGMENTS], scale_from[SEGMENTS];
    const int64_t base_a = GROUPED ? 0 : first, base_b = matrix * p.rows_b + first_wt;
    const uint8_t *const a_base = p.a + base_a * row_bytes, *const b_base = p.b + base_b * row_bytes;
    const uint8_t *const sa_base = (const uint8_t *)p.sa + base_a * scale_bytes, *const sb_base = (const uint8_t *)p.sb + base_b * scale_bytes;
#pragma unroll
    for (int s = 0; s < SEGMENTS; s++) {
        const int row = (wave * SEGMENTS + s) * 8 + (lane >> 3), piece = (lane & 7) ^ (lane >> 3);
        const int64_t r = row < TOK ? row_of_a(first + row) - base_a : row_of_b(first_wt + row - TOK) - first_wt;
        from[s] = (Offset)(r * row_bytes + piece * 16);
        scale_from[s] = (Offset)(r * scale_bytes);
    }
    const int n = (int)p.kb;
    const auto bring = [&](int kb, uint8_t *stage) {
#pragma unroll
        for (int l = 0; l < SEGMENTS; l++) {
            const int segment = wave * SEGMENTS + l;
            asm volatile("" : "+v"(from[l]));                     // (else its sum with the base is kept, in twice the registers)
            to_lds((segment * 8 < TOK ? a_base : b_base) + (int64_t)kb * RUN4_BYTES, from[l], stage + segment * 1024);
        }
    };
    // half of a wave's scales of four runs (a lane has four bytes; past the last run: the last four again)
    const auto bring_scales = [&](int group, int half) {
        const int row = wave * SEGMENTS * 8 + (lane >> 3);        // (its bits 2 and 3 are those of all its segments but for the segment's own)
#pragma unroll
        for (int l = half * SEGMENTS / 2; l < (half + 1) * SEGMENTS / 2; l++) {
            const int segment = wave * SEGMENTS + l, which = (lane & 7) ^ ((row + l * 8) >> 2 & 3) * 2;
            asm volatile("" : "+v"(scale_from[l]));
            to_lds4((segment * 8 < TOK ? sa_base : sb_base), scale_from[l] + 4 * (uint32_t)min(group * ROUND * 2 + which, 2 * n - 1), scales[group & 1] + segment * 256);
        }
    };

    v4f sum[I][J];
#pragma unroll
    for (int i = 0; i < I; i++)
#pragma unroll
        for (int j = 0; j < J; j++) sum[i][j] = {0.0f, 0.0f, 0.0f, 0.0f};

    const int low = ((lane >> 4) ^ (lane & 7)) * 16, byte = (lane >> 4) * 8;
    const int at_a = (wave_tok + (lane & 15)) * RUN4_BYTES + low, at_w = (TOK + wave_wt + (lane & 15)) * RUN4_BYTES + low;
    const auto operand = [&](const uint8_t *stage, int at, int half, int piece) { return *(const v4i *)(stage + (at ^ half * 64) + piece * 16 * RUN4_BYTES); };
    // Step N of a round of four multiplies a run and fills the stage that was multiplied before it with the run STAGES - 1 further on (the last run once more where
    // there is none left); the first two bring the next round's scales.  Before that a wave's loads of this run and of its round's scales have arrived, those of
    // later runs need not have, and all waves are done with the stage that is filled.  Sixteen rows of b are read from the LDS while those before are
    // multiplied, and the second half's rows of a during the first half.
    uint8_t *const stages[4] = {stage0, stage1, stage2, stage3};
    const auto step = [&](int kb, auto at) {
        constexpr int N = decltype(at)::value, FREE = (N + STAGES - 1) % STAGES;
        constexpr int FLYING = STAGES == 2 ? 0 : 2 * SEGMENTS + (N == 1 || N == 3 ? SEGMENTS / 2 : N == 2 ? SEGMENTS : 0);       // loads of the two steps before
        const uint8_t *const stage = stages[N % STAGES];
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((FLYING & 15) | 7 << 4 | FLYING >> 4 << 14);       // (vmcnt, and lgkmcnt to zero)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (all of the run's scales before the next are asked for: the compiler does not tell their places apart and would wait for those)
        const uint8_t *const of = scales[kb / ROUND & 1] + ((N ^ ((lane & 15) >> 2)) * 8) + (lane & 15) * 32;
        uint2 sa[J], sb[I];
#pragma unroll
        for (int j = 0; j < J; j++) sa[j] = *(const uint2 *)(of + (wave_tok + j * 16) * 32);
#pragma unroll
        for (int i = 0; i < I; i++) sb[i] = *(const uint2 *)(of + (TOK + wave_wt + i * 16) * 32);
        v4i a[2][J], after = operand(stage, at_w, 0, 0);
#pragma unroll
        for (int j = 0; j < J; j++) a[0][j] = operand(stage, at_a, 0, j);
        bring(min(kb + STAGES - 1, n - 1), stages[FREE]);
        if constexpr (N < 2) bring_scales(kb / ROUND + 1, N);
#pragma unroll
        for (int q = 0; q < 2 * I; q++) {
            const int half = q / I, i = q % I;
            const v4i w = after;
            if (q + 1 < 2 * I) after = operand(stage, at_w, (q + 1) / I, (q + 1) % I);
            if (half == 0)
#pragma unroll
                for (int j = i * J / I; j < (i + 1) * J / I; j++) a[1][j] = operand(stage, at_a, 1, j);
            const uint32_t of_w = (half ? sb[i].y : sb[i].x) >> byte;
#pragma unroll
            for (int j = 0; j < J; j++) sum[i][j] = four_product(w, of_w, a[half][j], (half ? sa[j].y : sa[j].x) >> byte, sum[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    bring_scales(0, 0);
    bring_scales(0, 1);
#pragma unroll
    for (int m = 0; m < STAGES - 1; m++) bring(min(m, n - 1), stages[m]);
    int kb = 0;
    for (; kb + ROUND - 1 < n; kb += ROUND) {
        step(kb, One<0>());
        step(kb + 1, One<1>());
        step(kb + 2, One<2>());
        step(kb + 3, One<3>());
    }
    if (kb < n) step(kb, One<0>());
    if (kb + 1 < n) step(kb + 1, One<1>());
    if (kb + 2 < n) step(kb + 2, One<2>());
    // (the last steps brought the last run once more: to stages that results go to now, so it has to be there before any wave's barrier)
    __builtin_amdgcn_s_waitcnt(7 << 4);
    __syncthreads();

    // Out through the LDS, sixteen rows of a at a time, in whole lines
    typedef typename Out::T T;
    constexpr int ROW = I * 16 * sizeof(T), PITCH = ROW + 16, PER_ROW = ROW / 16, ROWS = 64 / PER_ROW;       // bytes; lanes of a row, rows of an instruction
    T *out = (T *)p.out;
    constexpr int HALF = (WAVES + 1) / 2;
    static_assert(HALF * 16 * PITCH <= BYTES, "");
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
        for (int m = 0; m < 16 / ROWS; m++) {
            const int row = m * ROWS + lane / PER_ROW, at = lane % PER_ROW * 16;
            const int64_t r = first + wave_tok + j * 16 + row, c = first_wt + wave_wt + at / sizeof(T);
            const v4i v = *(const v4i *)(mine + row * PITCH + at);
            if (r < end) store16<T>(out + r * p.stride + c, p.rows_b - c, wide, v);
        }
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
    }
}

// ---- few rows -----------------------------------------------------------------------------------------------------
// The weights go from memory to registers, sixteen rows of a run of 256 columns a wave.  A workgroup takes STRIPS times sixteen rows of b, and as many of
// its eight waves share the runs of each.  Rows of a, J times sixteen, come from the caches.  RAW ones, up to sixteen, are brought to 4 bits by the
// workgroup, CHUNK runs at a time, while the first weights are on their way, and handed round through the LDS (by every wave for itself: 27.7 us where 10.7 do for 120 rows of
// 100 experts of 1000 x 1100).  Where the weights are few a workgroup's own chain bounds it (x, its 4 bits,
// a barrier, the waves' sums): of a run of launches one row times 4096 x 4096 takes 4.9 us, 3.8 where the last cache has the weights, and 3.5 with one strip of them alone, of which
// a launch that writes one number is 1.6.  Memory does where they are many: 8192 x 8192 10.7 us, 3.3 TB/s.
constexpr int FEW4_WAVES = 8;

// grid: groups of strips of sixteen rows of b, tiles of 16 * J rows of a
template <class In, int J, int STRIPS, class Out> __global__ __launch_bounds__(64 * FEW4_WAVES) void product_four_few_kernel(ProductArgs p, bool wide)
{
    constexpr bool RAW = !std::is_same<In, void>::value;
    constexpr int SHARE = FEW4_WAVES / STRIPS, AHEAD = STRIPS == 1 ? 2 : 4, CHUNK = 16, PITCH = RUN4_BYTES + 16;
    typedef Parts<4> P;
    __shared__ v4f parts[FEW4_WAVES][J][64];
    __shared__ __align__(16) uint8_t columns[RAW ? CHUNK * 16 * PITCH : 16], scales[RAW ? CHUNK * 16 * RUN4_SCALES : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t strip = (int64_t)blockIdx.x * STRIPS + wave % STRIPS;
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
    const int64_t r = strip * 16 + tok, row_b = matrix * p.rows_b + (r < p.rows_b ? r : p.rows_b - 1);
    const uint8_t *b = p.b + row_b * p.kb * RUN4_BYTES + quarter * 16, *sb = (const uint8_t *)p.sb + row_b * p.kb * RUN4_SCALES;
    const int byte = quarter * 8, kb = (int)p.kb;                 // of four scales, the lane's (a load of all eight of a run costs half of what two of a byte do)
    v4f sum[J];
#pragma unroll
    for (int j = 0; j < J; j++) sum[j] = {0.0f, 0.0f, 0.0f, 0.0f};
    v4i w[AHEAD][2];
    uint2 of_b[AHEAD];
    const auto fetch = [&](int run0, int end_run) {
#pragma unroll
        for (int n = 0; n < AHEAD; n++) {
            const int run = run0 + n * SHARE;
            if (run >= end_run) break;
            of_b[n] = *(const uint2 *)(sb + (int64_t)run * RUN4_SCALES);
#pragma unroll
            for (int half = 0; half < 2; half++) w[n][half] = *(const v4i *)(b + (int64_t)run * RUN4_BYTES + half * 64);
        }
    };
    const auto use = [&](int run0, int end_run, int chunk) {
#pragma unroll
        for (int n = 0; n < AHEAD; n++) {
            const int run = run0 + n * SHARE;
            if (run >= end_run) break;
#pragma unroll
            for (int j = 0; j < J; j++) {
                const int64_t at = RAW ? (run - chunk) * 16 + tok : src[j] * kb + run;
                const uint8_t *values = RAW ? columns + at * PITCH + quarter * 16 : p.a + at * RUN4_BYTES + quarter * 16;
                const v4i a0 = *(const v4i *)values, a1 = *(const v4i *)(values + 64);
                const uint2 of_a = *(const uint2 *)((RAW ? scales : (const uint8_t *)p.sa) + at * RUN4_SCALES);
                sum[j] = four_product(w[n][0], of_b[n].x >> byte & 255, a0, of_a.x >> byte & 255, sum[j]);
                sum[j] = four_product(w[n][1], of_b[n].y >> byte & 255, a1, of_a.y >> byte & 255, sum[j]);
            }
        }
    };
    const int mine = wave / STRIPS;
    if constexpr (RAW) {
        const int rows = (int)min(end - first, (int64_t)16), part = lane & 31;
        for (int chunk = 0; chunk < kb; chunk += CHUNK) {
            const int end_run = min(chunk + CHUNK, kb);
            fetch(chunk + mine, end_run);
            if (chunk > 0) __syncthreads();
            for (int i = (int)threadIdx.x >> 5; i < (end_run - chunk) * rows; i += FEW4_WAVES * 2) {
                const int run = i / rows, row = i - run * rows;
                float v[8];
                eight_of((const typename In::T *)p.a + __shfl(src[0], row) * p.stride_raw, (int64_t)(chunk + run) * RUN4 + part * 8, p.cols, v);
                uint32_t scale;
                *(uint32_t *)(columns + (run * 16 + row) * PITCH + part * 4) = P::to(v, scale);
                P::put_scale(scales + (run * 16 + row) * RUN4_SCALES, part, scale);
            }
            __syncthreads();
            for (int run0 = chunk + mine; run0 < end_run; run0 += SHARE * AHEAD) {
                use(run0, end_run, chunk);
                fetch(run0 + SHARE * AHEAD, end_run);
            }
        }
    } else
        for (int run0 = mine; run0 < kb; run0 += SHARE * AHEAD) {
            fetch(run0, kb);
            use(run0, kb, 0);
        }
#pragma unroll
    for (int j = 0; j < J; j++) parts[wave][j][lane] = sum[j];
    __syncthreads();
    for (int n = wave; n < J * STRIPS; n += FEW4_WAVES) {
        const int j = n / STRIPS, which = n % STRIPS;
        v4f total = parts[which][j][lane];
#pragma unroll
        for (int w = 1; w < SHARE; w++) total += parts[w * STRIPS + which][j][lane];
        const int64_t row = first + j * 16 + tok, c = ((int64_t)blockIdx.x * STRIPS + which) * 16 + quarter * 4;
        if (row < end) store_four<Out>((typename Out::T *)p.out + row * p.stride + c, p.rows_b - c, wide, total);
    }
}

// places in use by `slots` slots of E experts, each expert's rounded up to whole tiles: what there can be at most
int64_t most_tiles4(int64_t slots, int64_t E, int rows) { return slots / rows + (slots < E ? slots : E); }

bool grouped4(const ProductArgs &p) { return p.mode == ASGD_PRODUCT_GATHER || p.mode == ASGD_PRODUCT_PLACES; }

// rows of a (of an expert, on average)
int64_t rows_each4(const ProductArgs &p) { return grouped4(p) ? p.order.T * p.order.k / p.order.E : p.rows_a; }

// Four strips a workgroup (its rows of a, its place among the experts and its end are then there once for four) where that leaves more than a workgroup for
// each of the 256 compute units.
bool more_strips4(unsigned strips, unsigned tiles) { return (int64_t)strips * tiles >= 2048; }

}  // namespace

// Which tile: us of n tiles on 256 compute units, from what a tile's run takes with a unit to itself, what it takes among many, and what a tile takes
// besides, its results above all; all measured: 64 x 64 0.4, 0.21 and 0.8, 128 x 128 0.8, 0.55 and 1.8, 256 x 256 1.75, 1.75 and 8.9.  What each takes, and so what the rule
// decides between, in that order: 777 x 1001 x 1100 6.8, 10.0, 26.0; 256 x 4096 x 4096 10.2, 15.3, 30.6; 2048^3 13.6, 10.8, 19.2; 8192 x 8192 x 512 78, 46, 50;
// 4096^3 72.9, 44.3, 40.6; 8192^3 486, 310, 259 us.
static double tiles_time4(int64_t rows, int64_t outs, int64_t runs, int tile, double alone, double among, double once)
{
    const double rounds = (double)((((rows + tile - 1) / tile) * ((outs + tile - 1) / tile) + 255) / 256);
    return (double)runs * (alone > rounds * among ? alone : rounds * among) + rounds * once;
}

int product_four_form(const ProductArgs &p)
{
    if (rows_each4(p) <= 32) return ASGD_PRODUCT_FORM_FEW;
    if (grouped4(p)) return ASGD_PRODUCT_FORM_TILES_128;
    const double t64 = tiles_time4(p.rows_a, p.rows_b, p.kb, 64, 0.4, 0.21, 0.8), t128 = tiles_time4(p.rows_a, p.rows_b, p.kb, 128, 0.8, 0.55, 1.8);
    if (t64 < t128) return ASGD_PRODUCT_FORM_TILES_64;
    return tiles_time4(p.rows_a, p.rows_b, p.kb, 256, 1.75, 1.75, 8.9) < t128 ? ASGD_PRODUCT_FORM_TILES_256 : ASGD_PRODUCT_FORM_TILES_128;
}

hipError_t launch_product_four(const ProductArgs &p, int type, hipStream_t s)
{
    const bool grouped = grouped4(p);
    const int form = product_four_form(p);
    const bool wide4 = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * type_size(type)) == 0;
    const bool wide16 = p.stride * type_size(type) % 16 == 0 && (uintptr_t)p.out % 16 == 0;
    const auto tiles_of = [&](int tok) { return grouped ? most_tiles4(p.order.T * p.order.k, p.order.E, tok) : (p.rows_a + tok - 1) / tok; };
    return with_type(type, [&](auto out) {
        typedef decltype(out) Out;
        const auto few = [&](auto j) {
            constexpr int J = decltype(j)::value;
            const unsigned strips = (unsigned)((p.rows_b + 15) / 16), tiles = (unsigned)tiles_of(16 * J);
            if (more_strips4(strips, tiles)) product_four_few_kernel<void, J, 4, Out><<<dim3((strips + 3) / 4, tiles), 64 * FEW4_WAVES, 0, s>>>(p, wide4);
            else product_four_few_kernel<void, J, 1, Out><<<dim3(strips, tiles), 64 * FEW4_WAVES, 0, s>>>(p, wide4);
            return hipGetLastError();
        };
        const auto tiles = [&](auto tok, auto wt, auto waves_tok, auto waves_wt, auto stages, auto by_expert) {
            constexpr int TOK = decltype(tok)::value, WT = decltype(wt)::value, WAVES = decltype(waves_tok)::value * decltype(waves_wt)::value;
            const int64_t tiles_tok = tiles_of(TOK), tiles_wt = (p.rows_b + WT - 1) / WT;
            product_four_kernel<TOK, WT, decltype(waves_tok)::value, decltype(waves_wt)::value, decltype(stages)::value, decltype(by_expert)::value, Out>
                <<<(unsigned)(tiles_tok * tiles_wt), 64 * WAVES, 0, s>>>(p, (uint32_t)tiles_tok, (uint32_t)tiles_wt, wide16);
            return hipGetLastError();
        };
        if (form == ASGD_PRODUCT_FORM_FEW) return rows_each4(p) <= 16 ? few(One<1>()) : few(One<2>());
        if (grouped) return tiles(One<128>(), One<128>(), One<2>(), One<4>(), One<2>(), std::true_type());
        if (form == ASGD_PRODUCT_FORM_TILES_64) return tiles(One<64>(), One<64>(), One<2>(), One<2>(), One<4>(), std::false_type());
        if (form == ASGD_PRODUCT_FORM_TILES_256) return tiles(One<256>(), One<256>(), One<4>(), One<2>(), One<2>(), std::false_type());
        return tiles(One<128>(), One<128>(), One<2>(), One<4>(), One<2>(), std::false_type());
    });
}

hipError_t launch_product_four_raw(const ProductArgs &p, int raw_type, int type, hipStream_t s)
{
    const bool wide = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * type_size(type)) == 0;
    const unsigned strips = (unsigned)((p.rows_b + 15) / 16), tiles = grouped4(p) ? (unsigned)most_tiles4(p.order.T * p.order.k, p.order.E, 16) : 1u;
    return with_type(raw_type, [&](auto in) {
        return with_type(type, [&](auto out) {
            if (more_strips4(strips, tiles)) product_four_few_kernel<decltype(in), 1, 4, decltype(out)><<<dim3((strips + 3) / 4, tiles), 64 * FEW4_WAVES, 0, s>>>(p, wide);
            else product_four_few_kernel<decltype(in), 1, 1, decltype(out)><<<dim3(strips, tiles), 64 * FEW4_WAVES, 0, s>>>(p, wide);
            return hipGetLastError();
        });
    });
}

}  // namespace asgd
