// Launch interface of the layers (kavg_group_norm, kavg_dropout) and what their kernels share.  The boundary (layers_api.hip) has
// checked every argument; launchers derive grids.
#pragma once
#include "kavg_internal.h"
#include "counter_stream.h"

namespace kavg {

// which elements are dropped, and by what the others are multiplied
struct DropRule {
    uint64_t base;        // seed + (1 + site 2^40) gamma
    uint32_t threshold;   // 0: none is dropped; 65536: all
    float scale;
};
DropRule drop_rule(double drop, uint64_t seed, uint64_t site);

struct Strides { int64_t set, image, row; };

struct NormCall {
    int dtype, activation;
    int64_t sets, images, positions;
    int channels, groups;
    float eps;
    DropRule drop;
    const void* x; Strides xs;
    const void* dy; Strides dys;            // backward
    void* out; Strides outs;                // y, or dx
    const float* weight; int64_t weight_stride;
    const float* bias; int64_t bias_stride;
    float* mean; float* rstd;               // written by the forward pass (or null), read by the backward pass
    float* dweight; int64_t dweight_stride; // backward, or null
    float* dbias; int64_t dbias_stride;
};

hipError_t launch_group_norm(const NormCall& c, hipStream_t st);
hipError_t launch_group_norm_backward(const NormCall& c, hipStream_t st);

struct DropCall {
    int dtype;
    const void* x; int64_t x_stride;
    const void* residual; int64_t residual_stride;   // or null
    void* y; int64_t y_stride;
    int64_t rows, cols;
    DropRule drop;
};
hipError_t launch_dropout(const DropCall& c, hipStream_t st);

#if defined(__HIPCC__)
// 64 bits for the four elements 4q .. 4q+3
__device__ __forceinline__ uint64_t drop_bits(const DropRule& d, uint64_t q) { return splitmix64_mix(d.base + q * SPLITMIX_GAMMA); }
__device__ __forceinline__ bool drop_keeps(const DropRule& d, uint64_t e) {
    return (uint32_t)(drop_bits(d, e >> 2) >> (16 * (e & 3)) & 0xFFFF) >= d.threshold;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__bf16 v) { return (float)v; }
template <class E> __device__ __forceinline__ E from_float(float v) { return (E)v; }     // bf16: nearest, ties to even

// 1 / (1 + exp(-z)) with the hardware's exponential and reciprocal: a relative error of a few 2^-24 (z times log2 e is rounded once
// before the exponential, so up to |z| 2^-24 more)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f)); }

template <int ACT> __device__ __forceinline__ float activate(float z) {
    if (ACT == KAVG_ACT_RELU) return z < 0.f ? 0.f : z;             // (NaN stays)
    if (ACT == KAVG_ACT_SILU) return z * sigmoid(z);
    return z;
}
template <int ACT> __device__ __forceinline__ float activate_slope(float z) {
    if (ACT == KAVG_ACT_RELU) return z <= 0.f ? 0.f : 1.f;
    if (ACT == KAVG_ACT_SILU) { const float s = sigmoid(z); return s * (1.f + z * (1.f - s)); }
    return 1.f;
}
#endif

}  // namespace kavg
