// Group norm with an activation and dropout behind it, on channels-last images of several learners.  For a group (the D channels of
// a run at the S positions of an image), n = S D values:
//     m = mean x,  v = mean (x - m)^2,  r = (v + eps)^(-1/2),  xh = (x - m) r,  z = weight_c xh + bias_c,  y = drop(act(z)).
// Backward, with dz = act'(z) drop(dy) and h = weight_c dz:
//     dbias_c = sum dz,  dweight_c = sum dz xh  (over a learner's images and positions),
//     dx = r (h - mean h - xh mean(h xh))       (means over the group).
// Statistics and sums are fp32; the variance is taken about the mean, in a second sum.
#include "norm_tile.h"
#include "wave_sum.h"

namespace kavg {

namespace {

constexpr int T = 256;

// sum over the workgroup, the same in every thread
__device__ __forceinline__ float block_sum(float v, float* lds) {
    v = dpp_wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

struct Group { int64_t set, image; int group; };
__device__ __forceinline__ Group group_of_block(const NormCall& c) {
    const int64_t b = blockIdx.x, n = b / c.groups;
    return {n / c.images, n % c.images, (int)(b % c.groups)};
}

// one workgroup per group
template <class E, bool SILU>
__global__ void __launch_bounds__(T) norm_wide_forward_kernel(NormCall c) {
    __shared__ float lds[4];
    const Group at = group_of_block(c);
    const int D = c.channels / c.groups, c0 = at.group * D;
    const int64_t n = c.positions * D;
    const E* x = (const E*)c.x + at.set * c.xs.set + at.image * c.xs.image + c0;
    E* y = (E*)c.out + at.set * c.outs.set + at.image * c.outs.image + c0;
    float sum = 0.f;
    for (int64_t i = threadIdx.x; i < n; i += T) sum += to_float(x[i / D * c.xs.row + i % D]);
    const float mean = n ? block_sum(sum, lds) / (float)n : 0.f;
    sum = 0.f;
    for (int64_t i = threadIdx.x; i < n; i += T) { const float d = to_float(x[i / D * c.xs.row + i % D]) - mean; sum += d * d; }
    const float rstd = 1.f / sqrtf((n ? block_sum(sum, lds) / (float)n : 0.f) + c.eps);
    if (c.mean && threadIdx.x == 0) { c.mean[blockIdx.x] = mean; c.rstd[blockIdx.x] = rstd; }
    const uint64_t first = (uint64_t)(at.set * c.images + at.image) * c.positions * c.channels + c0;
    for (int64_t i = threadIdx.x; i < n; i += T) {
        const int64_t s = i / D;
        const int d = (int)(i % D), ch = c0 + d;
        const float xh = (to_float(x[s * c.xs.row + d]) - mean) * rstd;
        const float z = xh * (c.weight ? c.weight[at.set * c.weight_stride + ch] : 1.f) + (c.bias ? c.bias[at.set * c.bias_stride + ch] : 0.f);
        float a = SILU ? SILU_BACK * activate<true>(SILU_SCALE * z, 0.f) : activate<false>(z, c.floor);
        if (c.drop.threshold) a = drop_keeps(c.drop, first + (uint64_t)s * c.channels + d) ? a * c.drop.scale : 0.f;
        y[s * c.outs.row + d] = from_float<E>(a);
    }
}

template <class E, bool SILU>
__device__ __forceinline__ float grad_z(const NormCall& c, float dy, float z, uint64_t e) {
    if (c.drop.threshold) dy = drop_keeps(c.drop, e) ? dy * c.drop.scale : 0.f;
    return through_slope<SILU>(dy, SILU ? SILU_SCALE * z : z, c.floor);
}

// dx: one workgroup per group
template <class E, bool SILU>
__global__ void __launch_bounds__(T) norm_wide_backward_kernel(NormCall c) {
    __shared__ float lds[4];
    const Group at = group_of_block(c);
    const int D = c.channels / c.groups, c0 = at.group * D;
    const int64_t n = c.positions * D;
    const E* x = (const E*)c.x + at.set * c.xs.set + at.image * c.xs.image + c0;
    const E* dy = (const E*)c.dy + at.set * c.dys.set + at.image * c.dys.image + c0;
    E* dx = (E*)c.out + at.set * c.outs.set + at.image * c.outs.image + c0;
    const float mean = c.mean[blockIdx.x], rstd = c.rstd[blockIdx.x];
    const uint64_t first = (uint64_t)(at.set * c.images + at.image) * c.positions * c.channels + c0;
    float sh = 0.f, shx = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
        for (int64_t i = threadIdx.x; i < n; i += T) {
            const int64_t s = i / D;
            const int d = (int)(i % D), ch = c0 + d;
            const float w = c.weight ? c.weight[at.set * c.weight_stride + ch] : 1.f;
            const float xh = (to_float(x[s * c.xs.row + d]) - mean) * rstd;
            const float z = xh * w + (c.bias ? c.bias[at.set * c.bias_stride + ch] : 0.f);
            const float h = w * grad_z<E, SILU>(c, to_float(dy[s * c.dys.row + d]), z, first + (uint64_t)s * c.channels + d);
            if (pass == 0) { sh += h; shx += h * xh; }
            else dx[s * c.outs.row + d] = from_float<E>(rstd * (h - sh - xh * shx));
        }
        if (pass == 0) { sh = block_sum(sh, lds) / (float)n; shx = block_sum(shx, lds) / (float)n; }
    }
}

// dweight, dbias: one workgroup per learner and channel
template <class E, bool SILU>
__global__ void __launch_bounds__(T) norm_wide_param_kernel(NormCall c) {
    __shared__ float lds[4];
    const int64_t j = blockIdx.x / c.channels;
    const int ch = (int)(blockIdx.x % c.channels), g = ch / (c.channels / c.groups);
    const E* x = (const E*)c.x + j * c.xs.set + ch;
    const E* dy = (const E*)c.dy + j * c.dys.set + ch;
    const float w = c.weight ? c.weight[j * c.weight_stride + ch] : 1.f, b = c.bias ? c.bias[j * c.bias_stride + ch] : 0.f;
    float sz = 0.f, szx = 0.f;
    for (int64_t r = threadIdx.x; r < c.images * c.positions; r += T) {
        const int64_t i = r / c.positions, s = r % c.positions, stat = (j * c.images + i) * c.groups + g;
        const float xh = (to_float(x[i * c.xs.image + s * c.xs.row]) - c.mean[stat]) * c.rstd[stat];
        const uint64_t e = (uint64_t)((j * c.images + i) * c.positions + s) * c.channels + ch;
        const float dz = grad_z<E, SILU>(c, to_float(dy[i * c.dys.image + s * c.dys.row]), xh * w + b, e);
        sz += dz;
        szx += dz * xh;
    }
    sz = block_sum(sz, lds);
    szx = block_sum(szx, lds);
    if (threadIdx.x == 0) {
        if (c.dweight) c.dweight[j * c.dweight_stride + ch] = szx;
        if (c.dbias) c.dbias[j * c.dbias_stride + ch] = sz;
    }
}

template <class E, bool SILU>
hipError_t wide_backward(const NormCall& c, hipStream_t st) {
    const int64_t params = c.sets * c.channels, groups = c.sets * c.images * c.groups;
    if (c.dweight || c.dbias) norm_wide_param_kernel<E, SILU><<<dim3((unsigned)params), dim3(T), 0, st>>>(c);   // (before dx, which may be dy)
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && groups && c.positions) {
        norm_wide_backward_kernel<E, SILU><<<dim3((unsigned)groups), dim3(T), 0, st>>>(c);
        e = hipGetLastError();
    }
    return e;
}

hipError_t check(size_t want, const void* workspace, size_t bytes) {
    if (want > bytes) return hipErrorOutOfMemory;
    return want && (!workspace || ((uintptr_t)workspace & 15)) ? hipErrorInvalidValue : hipSuccess;
}

template <class E>
hipError_t backward(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    if (!c.sets) return hipSuccess;
    NormTiles t;
    const bool contiguous = c.xs.row == c.channels && c.dys.row == c.channels && c.outs.row == c.channels;
    if (c.images && c.positions && norm_tiles(c, contiguous, true, &t)) {
        const hipError_t e = check(norm_workspace(c, t, true), workspace, bytes);
        return e == hipSuccess ? tiled_backward<E>(c, t, workspace, st) : e;
    }
    return c.silu ? wide_backward<E, true>(c, st) : wide_backward<E, false>(c, st);
}

template <class E>
hipError_t forward(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    const int64_t groups = c.sets * c.images * c.groups;
    if (!groups) return hipSuccess;
    NormTiles t;
    const bool contiguous = c.xs.row == c.channels && c.outs.row == c.channels;
    if (c.positions && norm_tiles(c, contiguous, false, &t)) {
        const hipError_t e = check(norm_workspace(c, t, false), workspace, bytes);
        return e == hipSuccess ? tiled_forward<E>(c, t, workspace, st) : e;
    }
    const dim3 grid((unsigned)groups);
    if (c.silu) norm_wide_forward_kernel<E, true><<<grid, dim3(T), 0, st>>>(c);
    else norm_wide_forward_kernel<E, false><<<grid, dim3(T), 0, st>>>(c);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_group_norm(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    return c.dtype == KAVG_BF16 ? forward<__bf16>(c, workspace, bytes, st) : forward<float>(c, workspace, bytes, st);
}

hipError_t launch_group_norm_backward(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    return c.dtype == KAVG_BF16 ? backward<__bf16>(c, workspace, bytes, st) : backward<float>(c, workspace, bytes, st);
}

}  // namespace kavg
