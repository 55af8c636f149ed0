// Dropout from a counter-based generator: y = keep ? x / (1 - p) : 0, plus a residual.  The mask is a function of the element's number
// (counter_stream.h), so the backward pass draws it again and nothing is stored.  Bound by memory: an element is read and written once,
// and a draw of 64 bits serves four of them.
#include "layers.h"
#include <cmath>

namespace kavg {

DropRule drop_rule(double drop, uint64_t seed, uint64_t site) {
    const uint32_t t = (uint32_t)std::floor(drop * 65536 + 0.5);
    return {seed + (1 + (site << 40)) * SPLITMIX_GAMMA, t, t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.f};
}

namespace {

template <class E>
__global__ void __launch_bounds__(256) dropout_kernel(DropCall c) {
    const uint64_t n = (uint64_t)c.rows * c.cols;
    for (uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (uint64_t)gridDim.x * 256) {
        const uint64_t r = e / c.cols, k = e % c.cols;
        float v = drop_keeps(c.drop, e) ? to_float(((const E*)c.x)[r * c.x_stride + k]) * c.drop.scale : 0.f;
        if (c.residual) v += to_float(((const E*)c.residual)[r * c.residual_stride + k]);
        ((E*)c.y)[r * c.y_stride + k] = from_float<E>(v);
    }
}

}  // namespace

hipError_t launch_dropout(const DropCall& c, hipStream_t st) {
    const uint64_t n = (uint64_t)c.rows * c.cols;
    if (!n) return hipSuccess;
    const uint64_t blocks = (n + 255) / 256;
    const dim3 grid((unsigned)(blocks < (1u << 20) ? blocks : (1u << 20)));
    if (c.dtype == KAVG_BF16) dropout_kernel<__bf16><<<grid, dim3(256), 0, st>>>(c);
    else dropout_kernel<float><<<grid, dim3(256), 0, st>>>(c);
    return hipGetLastError();
}

}  // namespace kavg
