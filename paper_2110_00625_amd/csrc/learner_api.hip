// C entries of the products and of the step of learners whose local steps a caller writes: argument checks, then a launcher.  No state, no
// allocation, nothing that throws.
#include "adamw.h"
#include "linear.h"
#include <algorithm>
#include <cmath>

namespace {

using namespace kavg;

constexpr int64_t MOST_ROWS = INT32_MAX - 65535;             // (tiles reach past them in 32 bits)
constexpr int64_t MOST_COLUMNS = 1 << 27;                    // inputs, outputs: 2^21 tiles of 64; a launch takes 2^22
constexpr int64_t MOST_ELEMENTS = (int64_t)1 << 42, MOST_SPAN = (int64_t)1 << 46;

int64_t at_least_one(int64_t n) { return n > 1 ? n : 1; }
bool product_below(int64_t a, int64_t b, int64_t c, int64_t below) {
    const int64_t x = at_least_one(a), y = at_least_one(b), z = at_least_one(c);
    return x < below && y <= (below - 1) / x && z <= (below - 1) / (x * y);
}
// the stride of a dimension of one says nothing
bool stride_ok(int64_t stride, int64_t n, int64_t least) { return n < 2 || (stride >= least && stride <= MOST_SPAN / n); }

bool product_ok(const kavg_product* p) {
    if (!p || (p->dtype != KAVG_FP32 && p->dtype != KAVG_BF16) || p->activation < KAVG_ACT_NONE || p->activation > KAVG_ACT_SILU) return false;
    if (p->sets < 0 || p->rows < 0 || p->inputs < 1 || p->outputs < 1 || p->rows > MOST_ROWS || p->inputs > MOST_COLUMNS || p->outputs > MOST_COLUMNS) return false;
    return p->sets < (int64_t)1 << 31 && product_below(p->sets, p->rows, std::max(p->inputs, p->outputs), MOST_ELEMENTS) && product_below(p->sets, p->inputs, p->outputs, MOST_ELEMENTS);
}
bool empty(const kavg_product* p) { return !p->sets || !p->rows; }

bool rows_ok(const kavg_product* p, const kavg_rows* x, int64_t cols, bool written) {
    if (!x) return false;
    if (empty(p)) return true;
    if (!x->data || ((uintptr_t)x->data & (p->dtype == KAVG_BF16 ? 1 : 3))) return false;
    if (!stride_ok(x->row_stride, p->rows, written ? cols : 0) || !stride_ok(x->set_stride, p->sets, 0)) return false;
    if (!written || p->sets < 2) return true;
    // learners follow each other, or lie between each other's rows
    const int64_t rows = p->rows > 1 ? (p->rows - 1) * x->row_stride + cols : cols;
    return x->set_stride >= rows || (x->set_stride >= cols && (p->rows < 2 || x->row_stride >= (p->sets - 1) * x->set_stride + cols));
}

// [outputs][inputs] where inputs lie together (or there is one), else turned
bool turned(const kavg_product* p, const kavg_weights* w) { return p->inputs > 1 && w->input_stride != 1; }

bool weights_ok(const kavg_product* p, const kavg_weights* w, int elem, bool written) {
    if (!w) return false;
    if (!p->sets) return true;
    if (!w->data || ((uintptr_t)w->data & (elem - 1))) return false;
    const bool t = turned(p, w);
    const int64_t lines = t ? p->inputs : p->outputs, length = t ? p->outputs : p->inputs;
    if (t && p->outputs > 1 && w->output_stride != 1) return false;
    if (!stride_ok(t ? w->input_stride : w->output_stride, lines, written ? length : 0)) return false;
    const int64_t whole = lines > 1 ? (lines - 1) * (t ? w->input_stride : w->output_stride) + length : length;
    return stride_ok(w->set_stride, p->sets, written ? whole : 0);
}
Matrix matrix_of(const kavg_product* p, const kavg_weights* w) {
    const bool t = turned(p, w);
    const int64_t lines = t ? p->inputs : p->outputs, length = t ? p->outputs : p->inputs;
    return {w->data, p->sets > 1 ? w->set_stride : 0, lines > 1 ? (t ? w->input_stride : w->output_stride) : length};
}
Matrix matrix_of(const kavg_product* p, const kavg_rows* x, int64_t cols) {
    return {x->data, p->sets > 1 ? x->set_stride : 0, p->rows > 1 ? x->row_stride : cols};
}
bool vector_ok(const kavg_product* p, const float* v, int64_t stride, bool written) {
    return !((uintptr_t)v & 3) && (!v || stride_ok(stride, p->sets, written ? p->outputs : 0));
}
bool shares(const kavg_rows* a, const void* b) { return a && a->data == b; }

int status(hipError_t e) {
    return e == hipSuccess ? KAVG_OK : e == hipErrorOutOfMemory ? KAVG_ENOMEM : e == hipErrorInvalidValue ? KAVG_EINVAL : KAVG_EDEVICE;
}

ProductCall forward_of(const kavg_product* p) {
    ProductCall c = {};
    c.dtype = p->dtype; c.sets = p->sets;
    c.nR = (int)p->rows; c.nC = (int)p->outputs; c.nK = (int)p->inputs;
    c.finish.silu = p->activation == KAVG_ACT_SILU;
    c.finish.floor = p->activation == KAVG_ACT_RELU ? 0.f : -INFINITY;
    return c;
}
ProductCall inner_of(const kavg_product* p) {
    ProductCall c = {};
    c.dtype = p->dtype; c.sets = p->sets;
    c.nR = (int)p->rows; c.nC = (int)p->inputs; c.nK = (int)p->outputs;
    c.finish.slope_silu = p->activation == KAVG_ACT_SILU;
    c.finish.floor = -INFINITY;
    return c;
}

bool number_ok(double v) { return v >= 0. && std::isfinite(v); }
bool fp32_ok(double v) { return std::isfinite((float)v); }

}  // namespace

extern "C" {

int kavg_linear_workspace(const kavg_product* product, int backward, size_t* bytes) {
    if (!product_ok(product) || !bytes) return KAVG_EINVAL;
    *bytes = 0;
    if (empty(product)) return KAVG_OK;
    const int64_t sets = product->sets;
    const int rows = (int)product->rows, in = (int)product->inputs, out = (int)product->outputs, dtype = product->dtype;
    auto ask = [&](int nR, int nC, int nK, Turned turned) { *bytes = std::max(*bytes, product_plan(dtype, sets, nR, nC, nK, turned).bytes); };
    // (for weights and gradients in either order)
    for (const Turned turned : {NONE_TURNED, C_TURNED}) ask(rows, backward ? in : out, backward ? out : in, turned);
    if (backward) {
        ask(out, in, rows, BOTH_TURNED);
        ask(in, out, rows, BOTH_TURNED);
        ask(out, 0, rows, BOTH_TURNED);
    }
    return KAVG_OK;
}

int kavg_linear(const kavg_product* product, const kavg_rows* x, const kavg_weights* weight, const float* bias, int64_t bias_stride,
                const kavg_rows* residual, const kavg_rows* y, const kavg_rows* pre, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const kavg_product* p = product;
    if (!product_ok(p)) return KAVG_EINVAL;
    const int elem = p->dtype == KAVG_BF16 ? 2 : 4;
    if (!rows_ok(p, x, p->inputs, false) || !weights_ok(p, weight, elem, false) || !rows_ok(p, y, p->outputs, true)) return KAVG_EINVAL;
    if ((residual && !rows_ok(p, residual, p->outputs, false)) || (pre && !rows_ok(p, pre, p->outputs, true)) || !vector_ok(p, bias, bias_stride, false)) return KAVG_EINVAL;
    if (empty(p)) return KAVG_OK;
    if (shares(x, y->data) || weight->data == y->data || shares(pre, y->data) || shares(pre, x->data) || shares(pre, weight->data) || (residual && shares(pre, residual->data))) return KAVG_EINVAL;
    if (shares(residual, y->data) && ((p->rows > 1 && residual->row_stride != y->row_stride) || (p->sets > 1 && residual->set_stride != y->set_stride))) return KAVG_EINVAL;
    ProductCall c = forward_of(p);
    c.R = matrix_of(p, x, p->inputs);
    c.C = matrix_of(p, weight);
    c.c_turned = turned(p, weight);
    Finish& f = c.finish;
    f.bias = bias; f.bias_set = p->sets > 1 ? bias_stride : 0;
    if (pre) { const Matrix m = matrix_of(p, pre, p->outputs); f.kept = pre->data; f.kept_set = m.set_stride; f.kept_row = m.stride; }
    if (residual) { const Matrix m = matrix_of(p, residual, p->outputs); f.residual = residual->data; f.residual_set = m.set_stride; f.residual_row = m.stride; }
    const Matrix m = matrix_of(p, y, p->outputs);
    f.out = y->data; f.out_set = m.set_stride; f.out_row = m.stride;
    return status(launch_product(c, workspace, workspace_bytes, (hipStream_t)hip_stream));
}

int kavg_linear_backward(const kavg_product* product, const kavg_rows* dz, const kavg_rows* x, const kavg_weights* weight, const kavg_rows* pre,
                         const kavg_rows* dx, const kavg_weights* dweight, float* dbias, int64_t dbias_stride, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
    const kavg_product* p = product;
    if (!product_ok(p) || !rows_ok(p, dz, p->outputs, false)) return KAVG_EINVAL;
    const int elem = p->dtype == KAVG_BF16 ? 2 : 4;
    const bool slope = p->activation != KAVG_ACT_NONE;
    if (dx && (!rows_ok(p, dx, p->inputs, true) || !weights_ok(p, weight, elem, false) || (slope && !rows_ok(p, pre, p->inputs, false)))) return KAVG_EINVAL;
    if (dweight && (!rows_ok(p, x, p->inputs, false) || !weights_ok(p, dweight, 4, true))) return KAVG_EINVAL;
    if (!vector_ok(p, dbias, dbias_stride, true)) return KAVG_EINVAL;
    if (!empty(p) && dx && (shares(dx, dz->data) || dx->data == weight->data)) return KAVG_EINVAL;
    if (!empty(p) && dx && slope && shares(pre, dx->data) && ((p->rows > 1 && pre->row_stride != dx->row_stride) || (p->sets > 1 && pre->set_stride != dx->set_stride))) return KAVG_EINVAL;
    if (!p->sets) return KAVG_OK;
    const bool outer = dweight || dbias, inner = dx && p->rows;
    ProductCall w = {}, c = {};
    if (outer) {
        w.dtype = p->dtype; w.sets = p->sets;
        w.nK = (int)p->rows;
        w.r_turned = w.c_turned = true;
        w.finish.floor = -INFINITY;
        w.sums = dbias; w.sums_set = p->sets > 1 ? dbias_stride : 0;
        const Matrix of_dz = matrix_of(p, dz, p->outputs);
        const bool other = dweight && turned(p, dweight);                // dW lies as [inputs][outputs]
        if (other) {
            w.nR = (int)p->inputs; w.nC = (int)p->outputs;
            w.R = matrix_of(p, x, p->inputs); w.C = of_dz;
            w.side = dbias ? 2 : 0;
        } else {
            w.nR = (int)p->outputs; w.nC = dweight ? (int)p->inputs : 0;
            w.R = of_dz;
            if (dweight) w.C = matrix_of(p, x, p->inputs);
            w.side = dbias ? 1 : 0;
        }
        if (dweight) {
            const Matrix m = matrix_of(p, dweight);
            w.finish.out = dweight->data; w.finish.out_set = m.set_stride; w.finish.out_row = m.stride;
        }
    }
    if (inner) {
        c = inner_of(p);
        c.R = matrix_of(p, dz, p->outputs);
        c.C = matrix_of(p, weight);
        c.c_turned = !turned(p, weight);
        Finish& f = c.finish;
        if (slope) { const Matrix m = matrix_of(p, pre, p->inputs); f.before = pre->data; f.before_set = m.set_stride; f.before_row = m.stride; }
        const Matrix m = matrix_of(p, dx, p->inputs);
        f.out = dx->data; f.out_set = m.set_stride; f.out_row = m.stride;
    }
    // the weight gradient first: dx may lie where x does; but nothing if the block is too small for dx
    hipError_t e = inner && outer ? check_product(c, workspace, workspace_bytes) : hipSuccess;
    if (outer && e == hipSuccess) e = launch_product(w, workspace, workspace_bytes, (hipStream_t)hip_stream);
    if (inner && e == hipSuccess) e = launch_product(c, workspace, workspace_bytes, (hipStream_t)hip_stream);
    return status(e);
}

int kavg_adamw(const kavg_adamw_options* options, const kavg_adamw_tensor* tensors, int count, void* hip_stream) {
    const kavg_adamw_options* o = options;
    if (!o || (o->bits != 8 && o->bits != 32) || (o->grad_dtype != KAVG_FP32 && o->grad_dtype != KAVG_BF16)) return KAVG_EINVAL;
    if (!number_ok(o->lr) || !number_ok(o->eps) || !(o->beta1 >= 0. && o->beta1 < 1.) || !(o->beta2 >= 0. && o->beta2 < 1.) || !fp32_ok(o->lr) || !fp32_ok(o->grad_scale)) return KAVG_EINVAL;
    if ((!o->step && !o->step_dev) || count < 0 || (o->bits == 8 && count >= 1 << 24) || (count && !tensors)) return KAVG_EINVAL;
    if (((uintptr_t)o->step_dev & 7) || ((uintptr_t)o->lr_dev & 3) || ((uintptr_t)o->grad_scale_dev & 3)) return KAVG_EINVAL;
    const int grad_size = o->grad_dtype == KAVG_BF16 ? 2 : 4, state_size = o->bits / 8;
    for (int i = 0; i < count; ++i) {
        const kavg_adamw_tensor& t = tensors[i];
        if (t.rows < 0 || t.cols < 0 || t.reserved || !number_ok(t.weight_decay)) return KAVG_EINVAL;
        if (!t.rows || !t.cols) continue;
        if (t.rows >= (int64_t)1 << 31 || !product_below(t.rows, t.cols, 1, (int64_t)1 << 40)) return KAVG_EINVAL;
        if (!t.param || !t.grad || !t.m || !t.v || (o->bits == 8) != (t.m_scale != nullptr) || (o->bits == 8) != (t.v_scale != nullptr)) return KAVG_EINVAL;
        if (((uintptr_t)t.param & 3) || ((uintptr_t)t.grad & (grad_size - 1)) || (((uintptr_t)t.m | (uintptr_t)t.v) & (state_size - 1)) ||
            (((uintptr_t)t.m_scale | (uintptr_t)t.v_scale) & 3) || ((uintptr_t)t.copy & 1)) return KAVG_EINVAL;
        if (!stride_ok(t.param_stride, t.rows, t.cols) || !stride_ok(t.grad_stride, t.rows, 0) || (t.copy && !stride_ok(t.copy_stride, t.rows, t.cols))) return KAVG_EINVAL;
    }
    AdamwRule rule = {};
    rule.beta1 = (float)o->beta1; rule.rest1 = (float)(1. - o->beta1);
    rule.beta2 = (float)o->beta2; rule.rest2 = (float)(1. - o->beta2);
    rule.eps = (float)o->eps;
    rule.grad_scale = (float)o->grad_scale;
    rule.step = o->step; rule.seed = o->seed;
    rule.lr = o->lr; rule.exact1 = o->beta1; rule.exact2 = o->beta2; rule.exact_eps = o->eps;
    rule.wide = o->eps != 0. && (o->eps < 0x1p-126 || o->eps > 0x1p126);
    rule.step_dev = o->step_dev; rule.lr_dev = o->lr_dev; rule.grad_scale_dev = o->grad_scale_dev;
    return status(launch_adamw(o->bits, o->grad_dtype, rule, tensors, count, (hipStream_t)hip_stream));
}

}  // extern "C"
