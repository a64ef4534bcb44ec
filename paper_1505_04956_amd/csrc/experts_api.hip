// C entry points of the routed experts: what is refused, and which launch does the rest.
#include "four_bits.h"

using namespace asgd;

namespace {

constexpr int64_t MOST_ROWS = (int64_t)1 << 30;          // of an operand: byte offsets of its scales are 32-bit
constexpr int64_t MOST_COLS = (int64_t)1 << 24;
constexpr int64_t MOST_SLOTS = (int64_t)1 << 30;         // places are int32
constexpr int64_t MOST_GROUPS = (int64_t)1 << 23;        // workgroups of one launch

bool type_ok(int type) { return type == ASGD_TYPE_F32 || type == ASGD_TYPE_BF16 || type == ASGD_TYPE_F16; }
bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool matrix_ok(const void *p, int type, int64_t rows, int64_t cols, int64_t stride)
{
    return p && type_ok(type) && aligned(p, type_size(type)) && rows >= 0 && rows <= MOST_ROWS && cols >= 1 && cols <= MOST_COLS && (stride >= cols || rows <= 1) && stride >= 0 && stride <= ((int64_t)1 << 40);
}

bool rule_ok(const asgd_route_rule *r, int E)
{
    if (!r || E < 1 || E > ASGD_ROUTE_MAX_EXPERTS) return false;
    if (r->score != ASGD_SCORE_SOFTMAX && r->score != ASGD_SCORE_SIGMOID) return false;
    if (r->group_by != ASGD_GROUP_BEST && r->group_by != ASGD_GROUP_BEST_TWO) return false;
    if (r->groups < 1 || r->groups > ASGD_ROUTE_MAX_GROUPS || E % r->groups != 0 || r->kept < 1 || r->kept > r->groups) return false;
    const int width = E / r->groups;
    if (r->group_by == ASGD_GROUP_BEST_TWO && width < 2) return false;
    if (r->k < 1 || r->k > ASGD_ROUTE_MAX_CHOSEN || r->k > width * r->kept) return false;
    return (r->renormalize == 0 || r->renormalize == 1) && r->scale - r->scale == 0.0f;       // (a finite number)
}

bool order_ok(const asgd_route_order *o)
{
    return o && o->T >= 0 && o->k >= 1 && o->k <= ASGD_ROUTE_MAX_CHOSEN && o->E >= 1 && o->E <= ASGD_ROUTE_MAX_EXPERTS && o->T <= MOST_SLOTS / o->k &&
           o->offsets && o->blocks && (o->T == 0 || (o->slots && o->places)) && aligned(o->offsets, 4) && aligned(o->blocks, 4) && aligned(o->slots, 4) && aligned(o->places, 4);
}

bool blocks_ok(const asgd_blocks *m)
{
    if (!m || !m->values || m->rows < 0 || m->rows > MOST_ROWS || m->cols < 1 || m->cols > MOST_COLS || m->count < 1) return false;
    if (m->form == ASGD_BLOCKS_RAW) return m->count == 1 && matrix_ok(m->values, m->type, m->rows, m->cols, m->stride);
    if (m->form == ASGD_BLOCKS_FOURS) return m->scales && aligned(m->values, 16) && aligned(m->scales, 8) && m->count <= ASGD_ROUTE_MAX_EXPERTS;
    if (m->form != ASGD_BLOCKS_ROWS && m->form != ASGD_BLOCKS_SQUARES) return false;
    return m->scales && aligned(m->values, 16) && aligned(m->scales, 4) && (m->form == ASGD_BLOCKS_SQUARES || m->count == 1) && m->count <= ASGD_ROUTE_MAX_EXPERTS;
}

// A product but for its result: p and the rows of the result, or false.
bool product_ok(const asgd_blocks *a, const asgd_blocks *b, int mode, int exact, const asgd_route_order *order, ProductArgs &p, int64_t &out_rows)
{
    if (!blocks_ok(a) || !blocks_ok(b) || a->cols != b->cols || b->rows < 1 || b->rows > MOST_COLS || b->form == ASGD_BLOCKS_RAW || a->form == ASGD_BLOCKS_SQUARES || (exact != 0 && exact != 1))
        return false;
    const bool four = b->form == ASGD_BLOCKS_FOURS;
    if (four ? a->form != ASGD_BLOCKS_RAW && (a->form != ASGD_BLOCKS_FOURS || a->count != 1) : a->form == ASGD_BLOCKS_FOURS) return false;
    out_rows = a->rows;
    if (mode == ASGD_PRODUCT_ALL) {
        if (order || b->count != 1) return false;
    } else {
        if (!order_ok(order)) return false;
        const int64_t slots = order->T * order->k;
        if (mode == ASGD_PRODUCT_GATHER || mode == ASGD_PRODUCT_PLACES) {
            if ((b->form != ASGD_BLOCKS_SQUARES && !four) || b->count != order->E) return false;
            if (a->rows != (mode == ASGD_PRODUCT_GATHER ? order->T : slots)) return false;
            out_rows = slots;
        } else if (mode == ASGD_PRODUCT_OVER) {
            if (a->form != ASGD_BLOCKS_ROWS || b->form != ASGD_BLOCKS_ROWS || a->cols != BLOCK8 * asgd_route_max_blocks(order->T, order->k, order->E)) return false;
        } else return false;
    }
    p = {};
    p.a = (const uint8_t *)a->values; p.b = (const uint8_t *)b->values; p.sa = a->scales; p.sb = b->scales;
    p.rows_a = a->rows; p.rows_b = b->rows; p.kb = four ? runs4(a->cols) : blocks8(a->cols); p.cols = a->cols; p.mode = mode; p.exact = exact;
    if (order) p.order = *order;
    if (out_rows == 0) return true;
    if (a->form == ASGD_BLOCKS_RAW) {
        p.stride_raw = a->stride;
        return (b->form == ASGD_BLOCKS_SQUARES || four) && out_rows <= (mode == ASGD_PRODUCT_ALL ? ASGD_PRODUCT_RAW_ROWS : ASGD_PRODUCT_RAW_SLOTS) && (mode == ASGD_PRODUCT_ALL || mode == ASGD_PRODUCT_GATHER);
    }
    return !((double)blocks8(out_rows + (order ? (int64_t)BLOCK8 * order->E : 0)) * (mode == ASGD_PRODUCT_OVER ? order->E : 1) * blocks8(b->rows) > (double)(MOST_GROUPS / 2));      // (of 128 x 128: where thin, twice as many of 64 x 64)
}

// four neighbours of a row at a time
bool four_wide(const void *out, int type, int64_t stride) { return stride % 4 == 0 && aligned(out, 4 * type_size(type)); }

int done(hipError_t e) { return e == hipSuccess ? ASGD_OK : ASGD_EHIP; }

}  // namespace

extern "C" {

int asgd_route(const void *logits, int type, int64_t T, int E, int64_t stride, const float *bias, const asgd_route_rule *rule,
               int32_t *ids, float *weights, void *hip_stream)
{
    if (!rule_ok(rule, E) || !type_ok(type) || T < 0) return ASGD_EINVAL;
    if (T == 0) return ASGD_OK;
    if (!matrix_ok(logits, type, T, E, stride) || !ids || !weights || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(bias, 4)) return ASGD_EINVAL;
    RouteArgs a = {};
    a.logits = logits; a.bias = bias; a.ids = ids; a.weights = weights; a.T = T; a.stride = stride; a.E = E; a.rule = *rule;
    return done(launch_route(a, type, (hipStream_t)hip_stream));
}

int asgd_route_backward(const void *logits, int type, int64_t T, int E, int64_t stride, const float *bias,
                        const asgd_route_rule *rule, const int32_t *ids, const float *d_weights, void *d_logits,
                        int64_t d_stride, void *hip_stream)
{
    if (!rule_ok(rule, E) || !type_ok(type) || T < 0) return ASGD_EINVAL;
    if (T == 0) return ASGD_OK;
    if (!matrix_ok(logits, type, T, E, stride) || !matrix_ok(d_logits, type, T, E, d_stride) || !ids || !d_weights || !aligned(ids, 4) || !aligned(d_weights, 4) || !aligned(bias, 4))
        return ASGD_EINVAL;
    RouteArgs a = {};
    a.logits = logits; a.bias = bias; a.ids_in = ids; a.d_weights = d_weights; a.d_logits = d_logits; a.T = T; a.stride = stride; a.d_stride = d_stride;
    a.E = E; a.rule = *rule;
    return done(launch_route_backward(a, type, (hipStream_t)hip_stream));
}

size_t asgd_route_plan_bytes(int64_t T, int k, int E)
{
    if (T < 0 || k < 1 || k > ASGD_ROUTE_MAX_CHOSEN || E < 1 || E > ASGD_ROUTE_MAX_EXPERTS || T > MOST_SLOTS / k) return 0;
    return route_plan_bytes(T * k, E);
}

int asgd_route_plan(const int32_t *ids, const asgd_route_order *order, void *work, size_t work_bytes, void *hip_stream)
{
    if (!order_ok(order) || (order->T > 0 && !ids) || !aligned(ids, 4)) return ASGD_EINVAL;
    const size_t need = route_plan_bytes(order->T * order->k, order->E);
    if (need > 0 && (!work || work_bytes < need || !aligned(work, 16))) return ASGD_EINVAL;
    return done(launch_route_plan(ids, *order, work, (hipStream_t)hip_stream));
}

int64_t asgd_route_max_blocks(int64_t T, int k, int E)
{
    if (T < 0 || k < 1 || E < 1 || T > MOST_SLOTS / k) return 0;
    const int64_t slots = T * k;
    return slots / BLOCK8 + (slots < E ? slots : E);
}

int asgd_block_quantize(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, int turned,
                        const asgd_route_order *order, const float *weights, const asgd_blocks *out, void *hip_stream)
{
    if (!type_ok(type) || rows < 0 || !blocks_ok(out) || out->form == ASGD_BLOCKS_RAW || (turned != 0 && turned != 1)) return ASGD_EINVAL;
    if (out->form == ASGD_BLOCKS_FOURS && (turned || order)) return ASGD_EINVAL;
    if (order && (!order_ok(order) || out->form != ASGD_BLOCKS_ROWS || rows != order->T)) return ASGD_EINVAL;
    if (weights && (!order || !aligned(weights, 4))) return ASGD_EINVAL;
    const int64_t slots = order ? order->T * order->k : 0;
    const int64_t want_rows = turned ? cols : order ? slots : rows;
    const int64_t want_cols = !turned ? cols : order ? BLOCK8 * asgd_route_max_blocks(order->T, order->k, order->E) : rows;
    if (rows == 0) return ASGD_OK;
    if (!matrix_ok(x, type, rows, cols, stride) || (out->count > 1 && stride < cols)) return ASGD_EINVAL;
    if (out->rows != want_rows || out->cols != want_cols) return ASGD_EINVAL;
    if (out->form == ASGD_BLOCKS_FOURS) {
        if (rows * out->count > MOST_ROWS) return ASGD_EINVAL;
        const FourArgs f = {x, rows * out->count, cols, stride, (uint8_t *)out->values, (uint8_t *)out->scales};
        return done(launch_quantize_four(f, type, (hipStream_t)hip_stream));
    }
    QuantArgs q = {};
    q.x = x; q.rows = rows; q.cols = cols; q.stride = stride; q.count = out->count; q.values = (uint8_t *)out->values; q.scales = out->scales;
    q.out_rows = out->rows; q.out_blocks = blocks8(out->cols); q.weights = weights;
    if (order) q.order = *order;
    const hipStream_t s = (hipStream_t)hip_stream;
    if (out->form == ASGD_BLOCKS_SQUARES) {
        if ((double)blocks8(out->rows) * q.out_blocks * q.count > (double)MOST_GROUPS) return ASGD_EINVAL;
        return done(launch_quantize_squares(q, type, turned, s));
    }
    if (turned && q.out_blocks > MOST_GROUPS) return ASGD_EINVAL;
    return done(turned ? launch_quantize_turned(q, type, s) : launch_quantize_rows(q, type, s));
}

int asgd_block_expand(const asgd_blocks *x, void *out, int type, int64_t stride, void *hip_stream)
{
    if (!type_ok(type) || !blocks_ok(x) || x->form != ASGD_BLOCKS_FOURS) return ASGD_EINVAL;
    if (x->rows == 0) return ASGD_OK;
    if (x->rows > MOST_ROWS / x->count || !matrix_ok(out, type, x->rows * x->count, x->cols, stride)) return ASGD_EINVAL;
    const FourArgs f = {out, x->rows * x->count, x->cols, stride, (uint8_t *)x->values, (uint8_t *)x->scales};
    return done(launch_expand_four(f, type, (hipStream_t)hip_stream));
}

int asgd_block_quantize_both(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, const asgd_route_order *order,
                             const float *weights, const asgd_blocks *out, const asgd_blocks *out_turned, void *hip_stream)
{
    if (!type_ok(type) || rows < 0 || !blocks_ok(out) || !blocks_ok(out_turned) || out->form != ASGD_BLOCKS_ROWS || out_turned->form != ASGD_BLOCKS_ROWS) return ASGD_EINVAL;
    if (order && (!order_ok(order) || rows != order->T)) return ASGD_EINVAL;
    if (weights && (!order || !aligned(weights, 4))) return ASGD_EINVAL;
    if (rows == 0) return ASGD_OK;
    if (!matrix_ok(x, type, rows, cols, stride)) return ASGD_EINVAL;
    if (out->rows != (order ? order->T * order->k : rows) || out->cols != cols || out_turned->rows != cols || out_turned->cols != (order ? BLOCK8 * asgd_route_max_blocks(order->T, order->k, order->E) : rows))
        return ASGD_EINVAL;
    QuantArgs q = {};
    q.x = x; q.rows = rows; q.cols = cols; q.stride = stride; q.count = 1; q.values = (uint8_t *)out_turned->values; q.scales = out_turned->scales;
    q.out_rows = out_turned->rows; q.out_blocks = blocks8(out_turned->cols); q.weights = weights;
    if (order) q.order = *order;
    if (q.out_blocks > MOST_GROUPS) return ASGD_EINVAL;
    return done(launch_quantize_both(q, *out, type, (hipStream_t)hip_stream));
}

int asgd_block_product(const asgd_blocks *a, const asgd_blocks *b, int mode, int exact, const asgd_route_order *order, void *out,
                       int type, int64_t stride, void *hip_stream)
{
    ProductArgs p;
    int64_t out_rows;
    if (!type_ok(type) || !product_ok(a, b, mode, exact, order, p, out_rows)) return ASGD_EINVAL;
    if (out_rows == 0) return ASGD_OK;
    if (!matrix_ok(out, type, out_rows, b->rows, stride) || (mode == ASGD_PRODUCT_OVER && stride < b->rows)) return ASGD_EINVAL;
    p.out = out; p.stride = stride;
    const hipStream_t s = (hipStream_t)hip_stream;
    if (b->form == ASGD_BLOCKS_FOURS) return done(a->form == ASGD_BLOCKS_RAW ? launch_product_four_raw(p, a->type, type, s) : launch_product_four(p, type, s));
    return done(a->form == ASGD_BLOCKS_RAW ? launch_product_raw(p, a->type, type, s) : launch_product(p, b->form == ASGD_BLOCKS_SQUARES, type, s));
}

int asgd_block_product_form(const asgd_blocks *a, const asgd_blocks *b, int mode, int exact, const asgd_route_order *order)
{
    ProductArgs p;
    int64_t out_rows;
    if (!product_ok(a, b, mode, exact, order, p, out_rows) || out_rows == 0) return ASGD_PRODUCT_FORM_NONE;
    if (b->form == ASGD_BLOCKS_FOURS && a->form != ASGD_BLOCKS_RAW) return product_four_form(p);
    return a->form == ASGD_BLOCKS_RAW ? ASGD_PRODUCT_FORM_FEW : product_form(p, b->form == ASGD_BLOCKS_SQUARES);
}

int asgd_experts_direct(const asgd_blocks *x, const int32_t *ids, const float *weights, int k, const asgd_blocks *w, int exact,
                        void *out, int type, int64_t stride, void *hip_stream)
{
    if (!blocks_ok(x) || x->form != ASGD_BLOCKS_RAW || !blocks_ok(w) || (w->form != ASGD_BLOCKS_SQUARES && w->form != ASGD_BLOCKS_FOURS) || w->cols != x->cols || w->rows < 1 || w->rows > MOST_COLS)
        return ASGD_EINVAL;
    if (x->rows > (w->form == ASGD_BLOCKS_FOURS ? ASGD_PRODUCT_RAW_SLOTS : ASGD_PRODUCT_RAW_ROWS)) return ASGD_EINVAL;
    if (k < 1 || k > ASGD_ROUTE_MAX_CHOSEN || !type_ok(type) || (exact != 0 && exact != 1)) return ASGD_EINVAL;
    if (x->rows == 0) return ASGD_OK;
    if (!ids || !weights || !aligned(ids, 4) || !aligned(weights, 4) || !matrix_ok(out, type, x->rows, w->rows, stride)) return ASGD_EINVAL;
    if (w->form == ASGD_BLOCKS_FOURS) {
        const DirectArgs a = {x->values, x->stride, x->cols, w->rows, (int)x->rows, k, w->count, ids, weights, *w, out, stride, four_wide(out, type, stride)};
        return done(launch_direct_four(a, x->type, type, (hipStream_t)hip_stream));
    }
    ProductArgs p = {};
    p.a = (const uint8_t *)x->values; p.b = (const uint8_t *)w->values; p.sb = w->scales; p.rows_a = x->rows; p.rows_b = w->rows;
    p.kb = blocks8(x->cols); p.cols = x->cols; p.stride_raw = x->stride; p.out = out; p.stride = stride; p.exact = exact;
    return done(launch_product_direct(p, ids, weights, k, w->count, x->type, type, (hipStream_t)hip_stream));
}

int asgd_experts_sum(const void *y, int y_type, int64_t n, int64_t y_stride, const asgd_route_order *order, const float *weights,
                     void *out, int type, int64_t stride, void *hip_stream)
{
    if (!order_ok(order) || !type_ok(y_type) || !type_ok(type) || n < 1) return ASGD_EINVAL;
    if (order->T == 0) return ASGD_OK;
    if (!matrix_ok(y, y_type, order->T * order->k, n, y_stride) || !matrix_ok(out, type, order->T, n, stride) || !aligned(weights, 4)) return ASGD_EINVAL;
    SumArgs a = {};
    a.y = y; a.n = n; a.y_stride = y_stride; a.order = *order; a.weights = weights; a.out = out; a.stride = stride;
    return done(launch_experts_sum(a, y_type, type, (hipStream_t)hip_stream));
}

int asgd_experts_sum_backward(const void *d_out, int type, int64_t stride, const void *y, int y_type, int64_t n, int64_t y_stride,
                              const asgd_route_order *order, float *d_weights, void *hip_stream)
{
    if (!order_ok(order) || !type_ok(y_type) || !type_ok(type) || n < 1) return ASGD_EINVAL;
    if (order->T == 0) return ASGD_OK;
    if (!matrix_ok(y, y_type, order->T * order->k, n, y_stride) || !matrix_ok(d_out, type, order->T, n, stride) || !d_weights || !aligned(d_weights, 4)) return ASGD_EINVAL;
    SumArgs a = {};
    a.y = y; a.d_out = d_out; a.n = n; a.y_stride = y_stride; a.order = *order; a.d_weights = d_weights; a.stride = stride;
    return done(launch_experts_sum_backward(a, y_type, type, (hipStream_t)hip_stream));
}

size_t asgd_experts_layer_bytes(int64_t rows, int k, int E, int64_t D, int64_t H)
{
    if (rows < 0 || rows > ASGD_PRODUCT_RAW_ROWS || k < 1 || k > ASGD_ROUTE_MAX_CHOSEN || E < 1 || E > ASGD_ROUTE_MAX_EXPERTS || D < 1 || D > MOST_COLS || H < 1 || H > MOST_COLS / 2) return 0;
    return layer_bytes(rows, k, E, D, H);
}

int asgd_experts_layer(const asgd_blocks *x, const void *logits, int logits_type, int64_t logits_stride, const float *bias,
                       const asgd_route_rule *rule, const asgd_blocks *up, const asgd_blocks *down, int activation, int32_t *ids,
                       float *weights, void *out, int type, int64_t stride, void *work, size_t work_bytes, void *hip_stream)
{
    if (!blocks_ok(x) || x->form != ASGD_BLOCKS_RAW || x->rows > ASGD_PRODUCT_RAW_ROWS || !blocks_ok(up) || !blocks_ok(down)) return ASGD_EINVAL;
    if ((up->form != ASGD_BLOCKS_SQUARES && up->form != ASGD_BLOCKS_FOURS) || down->form != up->form || down->count != up->count || up->cols != x->cols) return ASGD_EINVAL;
    if (down->rows < 1 || down->rows > MOST_COLS || up->rows > MOST_COLS || up->rows != 2 * down->cols || (activation != ASGD_ACTIVATION_SILU && activation != ASGD_ACTIVATION_GELU)) return ASGD_EINVAL;
    if (!rule_ok(rule, up->count) || !type_ok(logits_type) || !type_ok(type)) return ASGD_EINVAL;
    if (x->rows == 0) return ASGD_OK;
    if (!matrix_ok(logits, logits_type, x->rows, up->count, logits_stride) || !matrix_ok(out, type, x->rows, down->rows, stride)) return ASGD_EINVAL;
    if (!ids || !weights || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(bias, 4)) return ASGD_EINVAL;
    if (!work || !aligned(work, 16) || work_bytes < layer_bytes(x->rows, rule->k, up->count, x->cols, down->cols)) return ASGD_EINVAL;
    RouteArgs r = {};
    r.logits = logits; r.bias = bias; r.T = x->rows; r.stride = logits_stride; r.E = up->count; r.rule = *rule;
    LayerArgs a = {};
    a.x = x->values; a.x_stride = x->stride; a.D = x->cols; a.H = down->cols; a.N = down->rows; a.x_type = x->type; a.T = (int)x->rows; a.k = rule->k; a.E = up->count;
    a.activation = activation; a.up = *up; a.down = *down; a.ids = ids; a.weights = weights; a.out = out; a.out_stride = stride; a.wide_out = four_wide(out, type, stride);
    return done(launch_layer(a, r, logits_type, type, work, (hipStream_t)hip_stream));
}

}  // extern "C"
