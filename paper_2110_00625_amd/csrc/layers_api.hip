// C entries of the layers: argument checks, then a launcher.  No state, no allocation, nothing that throws.
#include "layers.h"
#include <algorithm>
#include <cmath>

namespace {

using namespace kavg;

constexpr int64_t MOST_ELEMENTS = (int64_t)1 << 42;
constexpr int MOST_CHANNELS = INT32_MAX - 65535;            // (counted in 32 bits by lanes, the last of which lie behind them)

// a * b * c * d below the limit, each factor from 0 on (a size of 0 leaves the others alone)
bool product_ok(int64_t a, int64_t b, int64_t c, int64_t d, int64_t below) {
    int64_t p = 1;
    for (const int64_t f : {a, b, c, d}) {
        if (f < 0) return false;
        if (f > 1 && p > (below - 1) / f) return false;
        p *= f > 1 ? f : 1;
    }
    return true;
}

bool drop_ok(double drop, uint64_t site) { return drop >= 0. && drop <= 1. && site < ((uint64_t)1 << 24); }

bool norm_ok(const kavg_norm* n) {
    if (!n || n->reserved || (n->dtype != KAVG_FP32 && n->dtype != KAVG_BF16)) return false;
    if (n->activation < KAVG_ACT_NONE || n->activation > KAVG_ACT_SILU) return false;
    if (n->channels < 1 || n->channels > MOST_CHANNELS || n->groups < 1 || n->channels % n->groups) return false;
    if (!product_ok(n->sets, n->images, n->positions, n->channels, MOST_ELEMENTS)) return false;
    if (!product_ok(n->sets, n->images, n->groups, 1, (int64_t)1 << 31) || !product_ok(n->sets, n->channels, 1, 1, (int64_t)1 << 31)) return false;
    return n->eps > 0.f && std::isfinite(n->eps) && drop_ok(n->drop, n->site);
}

bool empty(const kavg_norm* n) { return !n->sets || !n->images || !n->positions; }

bool images_ok(const kavg_norm* n, const kavg_images* x, bool written) {
    if (!x) return false;
    if (empty(n)) return true;
    if (!x->data || ((uintptr_t)x->data & (n->dtype == KAVG_BF16 ? 1 : 3))) return false;
    struct { int64_t stride, size; } d[3] = {{x->row_stride, n->positions}, {x->image_stride, n->images}, {x->set_stride, n->sets}};
    for (auto& i : d) {
        if (i.size < 2) i = {0, 1};                         // (its stride says nothing)
        if (i.stride < 0 || i.stride > ((int64_t)1 << 46) / i.size) return false;
    }
    if (!written) return true;
    // from the densest dimension on, each has to step over what the ones before it span (a dimension of one is no step)
    std::sort(d, d + 3, [](const auto& a, const auto& b) { return a.stride < b.stride; });
    int64_t run = n->channels;
    for (const auto& i : d) {
        if (i.size > 1 && i.stride < run) return false;
        run += (i.size - 1) * i.stride;
    }
    return true;
}

// (the stride of one learner's parameters says nothing)
bool params_ok(const kavg_norm* n, const float* p, int64_t stride, bool written) {
    if (!p || n->sets < 2) return !((uintptr_t)p & 3);
    return !((uintptr_t)p & 3) && stride >= (written ? n->channels : 0) && stride <= ((int64_t)1 << 46) / n->sets;
}

// strides of a dimension of one are never multiplied by more than zero; they are set to 0 so that no launcher looks at them
Strides strides_of(const kavg_norm* n, const kavg_images* x) {
    return {n->sets > 1 ? x->set_stride : 0, n->images > 1 ? x->image_stride : 0, n->positions > 1 ? x->row_stride : n->channels};
}

NormCall call_of(const kavg_norm* n, bool backward) {
    NormCall c = {};
    c.dtype = n->dtype;
    c.silu = n->activation == KAVG_ACT_SILU;
    c.floor = n->activation == KAVG_ACT_RELU ? 0.f : backward ? NAN : -INFINITY;
    c.sets = n->sets;
    c.images = n->images;
    c.positions = n->positions;
    c.channels = n->channels;
    c.groups = n->groups;
    c.eps = n->eps;
    c.drop = drop_rule(n->drop, n->seed, n->site);
    return c;
}

int status(hipError_t e) {
    return e == hipSuccess ? KAVG_OK : e == hipErrorOutOfMemory ? KAVG_ENOMEM : e == hipErrorInvalidValue ? KAVG_EINVAL : KAVG_EDEVICE;
}

}  // namespace

extern "C" {

int kavg_group_norm_workspace(const kavg_norm* norm, int backward, size_t* bytes) {
    if (!norm_ok(norm) || !bytes) return KAVG_EINVAL;
    *bytes = empty(norm) ? 0 : norm_workspace(call_of(norm, backward != 0), backward != 0);
    return KAVG_OK;
}

int kavg_group_norm(const kavg_norm* norm, const kavg_images* x, const float* weight, int64_t weight_stride, const float* bias,
                    int64_t bias_stride, const kavg_images* y, float* mean, float* rstd, void* workspace, size_t workspace_bytes,
                    void* hip_stream) {
    if (!norm_ok(norm) || !images_ok(norm, x, false) || !images_ok(norm, y, true) || !mean != !rstd) return KAVG_EINVAL;
    if (!params_ok(norm, weight, weight_stride, false) || !params_ok(norm, bias, bias_stride, false)) return KAVG_EINVAL;
    NormCall c = call_of(norm, false);
    c.x = x->data; c.xs = strides_of(norm, x);
    c.out = y->data; c.outs = strides_of(norm, y);
    c.weight = weight; c.weight_stride = weight_stride;
    c.bias = bias; c.bias_stride = bias_stride;
    c.mean = mean; c.rstd = rstd;
    return status(launch_group_norm(c, workspace, workspace_bytes, (hipStream_t)hip_stream));
}

int kavg_group_norm_backward(const kavg_norm* norm, const kavg_images* dy, const kavg_images* x, const float* mean, const float* rstd,
                             const float* weight, int64_t weight_stride, const float* bias, int64_t bias_stride, const kavg_images* dx,
                             float* dweight, int64_t dweight_stride, float* dbias, int64_t dbias_stride, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
    if (!norm_ok(norm) || !images_ok(norm, dy, false) || !images_ok(norm, x, false) || !images_ok(norm, dx, true)) return KAVG_EINVAL;
    if ((!mean || !rstd) && !empty(norm)) return KAVG_EINVAL;
    if (!params_ok(norm, weight, weight_stride, false) || !params_ok(norm, bias, bias_stride, false)) return KAVG_EINVAL;
    if (!params_ok(norm, dweight, dweight_stride, true) || !params_ok(norm, dbias, dbias_stride, true)) return KAVG_EINVAL;
    NormCall c = call_of(norm, true);
    c.x = x->data; c.xs = strides_of(norm, x);
    c.dy = dy->data; c.dys = strides_of(norm, dy);
    c.out = dx->data; c.outs = strides_of(norm, dx);
    c.weight = weight; c.weight_stride = weight_stride;
    c.bias = bias; c.bias_stride = bias_stride;
    c.mean = const_cast<float*>(mean); c.rstd = const_cast<float*>(rstd);
    c.dweight = dweight; c.dweight_stride = dweight_stride;
    c.dbias = dbias; c.dbias_stride = dbias_stride;
    return status(launch_group_norm_backward(c, workspace, workspace_bytes, (hipStream_t)hip_stream));
}

int kavg_dropout(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* y, int64_t y_stride, int64_t rows,
                 int64_t cols, int dtype, double drop, uint64_t seed, uint64_t site, void* hip_stream) {
    if (dtype != KAVG_FP32 && dtype != KAVG_BF16) return KAVG_EINVAL;
    if (cols < 1 || !product_ok(rows, cols, 1, 1, MOST_ELEMENTS) || !drop_ok(drop, site)) return KAVG_EINVAL;
    if (rows == 0) return KAVG_OK;
    const uintptr_t odd = dtype == KAVG_BF16 ? 1 : 3;
    if (!x || !y || (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)y) & odd)) return KAVG_EINVAL;
    if (rows > 1) {
        const int64_t most = ((int64_t)1 << 46) / rows;
        if (x_stride < 0 || x_stride > most || (residual && (residual_stride < 0 || residual_stride > most)) || y_stride < cols || y_stride > most)
            return KAVG_EINVAL;
        const bool apart = x_stride != cols || y_stride != cols || (residual && residual_stride != cols);
        if (apart && cols >= (int64_t)1 << 30) return KAVG_EINVAL;
    }
    const bool one = rows < 2;                              // (its strides say nothing)
    DropCall c = {dtype, x, one ? cols : x_stride, residual, one ? cols : residual_stride, y, one ? cols : y_stride, rows, cols, drop_rule(drop, seed, site)};
    return status(launch_dropout(c, (hipStream_t)hip_stream));
}

int kavg_dropout_backward(const void* dy, int64_t dy_stride, void* dx, int64_t dx_stride, int64_t rows, int64_t cols, int dtype, double drop,
                          uint64_t seed, uint64_t site, void* hip_stream) {
    return kavg_dropout(dy, dy_stride, nullptr, 0, dx, dx_stride, rows, cols, dtype, drop, seed, site, hip_stream);
}

}  // extern "C"
