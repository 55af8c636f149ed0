// Group norm with an activation and dropout behind it, on channels-last images of several learners.  For a group (the D channels of
// a run at the S positions of an image), n = S D values:
//     m = mean x,  v = mean (x - m)^2,  r = (v + eps)^(-1/2),  xh = (x - m) r,  z = weight_c xh + bias_c,  y = drop(act(z)).
// Backward, with dz = act'(z) drop(dy) and h = weight_c dz:
//     dbias_c = sum dz,  dweight_c = sum dz xh  (over a learner's images and positions),
//     dx = r (h - mean h - xh mean(h xh))       (means over the group).
// Statistics are fp32; the variance is taken about the mean, in a second sum.  Sums of any number of terms are 64 bits wide, of up to some
// hundred fp32.
//
// Most calls run on tiles in registers (norm_tile.h).  What no tile takes, groups wider than 8192 channels (fp32: 4096), odd ones of more than
// some hundred, and counts of tiles past 2^30, runs on the kernels here: a lane per channel goes along its chunk of the positions, sums per channel
// and chunk go through memory to the groups, and the image is read again for the results.  They are right for any size, load an element at a
// time (128 bytes of bf16 a wavefront, eight rows of them in flight), and are bound by that and by their launches' latencies: 8 images of 1000
// positions, 1031 channels in one group, in bf16, backward 53 us (a workgroup per group, for whom there are eight: 2475); 64 vectors of 16384
// forward 23, backward 33 (17 and 26).
#include "norm_backward.h"
#include "norm_forward.h"
#include "wave_sum.h"
#include <algorithm>

namespace kavg {

extern template hipError_t tiled_forward<float>(const NormCall&, const NormTiles&, void*, hipStream_t);
extern template hipError_t tiled_forward<__bf16>(const NormCall&, const NormTiles&, void*, hipStream_t);
extern template hipError_t tiled_backward<float>(const NormCall&, const NormTiles&, void*, hipStream_t);
extern template hipError_t tiled_backward<__bf16>(const NormCall&, const NormTiles&, void*, hipStream_t);

namespace {

constexpr int T = 256;
constexpr int ROWS = 8;                              // loads of a lane in flight
constexpr int64_t WIDE_GROUPS = 1024;                // workgroups wanted
constexpr int64_t MOST_GROUPS = 4096;                // of a launch

struct Chunks { int64_t rows; int count; };          // positions of a chunk

Chunks chunks_of(const NormCall& c) {
    const int64_t tiles = std::max<int64_t>(1, c.sets * c.images * ((c.channels + T - 1) / T));
    if (!c.positions) return {1, 0};
    const int64_t want = std::min(c.positions, (WIDE_GROUPS + tiles - 1) / tiles), rows = (c.positions + want - 1) / want;
    return {rows, (int)((c.positions + rows - 1) / rows)};
}

struct WideCall {
    NormCall n;
    int64_t rows;
    int chunks;
    float* parts;                                    // [image][chunk] of two sums per channel
    float *mean, *rstd;                              // forward: [image][group]
    const float* group_sums;                         // backward: [image][group] of (A, B)
};

// a lane's channel, and its chunk of an image's positions: workgroups along x, y, and z (which go on with further images)
struct WidePlace {
    int64_t image, row, rows;                        // image: of all learners'
    uint32_t set, in_set;
    int chunk, ch, group;
    bool on;
    __device__ __forceinline__ WidePlace(const WideCall& f, int64_t image) : image(image) {
        ch = blockIdx.x * T + threadIdx.x;
        on = ch < f.n.channels;
        group = on ? ch / (f.n.channels / f.n.groups) : 0;
        chunk = blockIdx.y;
        set = (uint32_t)image / (uint32_t)f.n.images;
        in_set = (uint32_t)image - set * (uint32_t)f.n.images;
        row = chunk * f.rows;
        rows = f.n.positions - row < f.rows ? f.n.positions - row : f.rows;
    }
    template <class E> __device__ __forceinline__ E* at(const void* p, const Strides& s) const { return (E*)p + set * s.set + in_set * s.image + row * s.row + ch; }
    __device__ __forceinline__ uint64_t number(const NormCall& c) const { return (uint64_t)(image * c.positions + row) * c.channels + ch; }
    __device__ __forceinline__ float* parts(const WideCall& f) const { return f.parts + (image * f.chunks + chunk) * 2 * f.n.channels + ch; }
};

// f(first, constant: how many) of rows of a chunk: ROWS at a time, then one
template <class F> __device__ __forceinline__ void for_rows(int64_t rows, F f) {
    int64_t s = 0;
    for (; s + ROWS <= rows; s += ROWS) f(s, std::integral_constant<int, ROWS>());
    for (; s < rows; ++s) f(s, std::integral_constant<int, 1>());
}

// mean and squared distances from it of a channel in a chunk, eight values at a time, joined as means of parts (in 64 bits: a chunk may be the whole
// image, of any length)
template <class E>
__global__ void __launch_bounds__(T) norm_wide_moments_kernel(WideCall f) {
    for (int64_t image = blockIdx.z; image < f.n.sets * f.n.images; image += gridDim.z) {
        const WidePlace l(f, image);
        if (!l.on) continue;
        const E* x = l.at<const E>(f.n.x, f.n.xs);
        double mean = 0., sq = 0.;
        for_rows(l.rows, [&](int64_t s, auto some) {
            constexpr int K = some.value;
            float v[K], sum = 0.f, q = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i) v[i] = to_float(x[(s + i) * f.n.xs.row]);
#pragma unroll
            for (int i = 0; i < K; ++i) sum += v[i];
            const float m = sum * (1.f / K);
#pragma unroll
            for (int i = 0; i < K; ++i) q += (v[i] - m) * (v[i] - m);
            const float d = (float)(m - mean), share = (float)K / (float)(s + K);
            mean += d * share;
            sq += q + d * d * ((float)s * share);
        });
        float* to = l.parts(f);
        to[0] = (float)mean;
        to[f.n.channels] = (float)sq;
    }
}

constexpr int JOIN = 1024;                           // lanes that join a group's channels and chunks

// sum over a workgroup of JOIN lanes, the same in every one
__device__ __forceinline__ float block_sum(float v, float* lds) {
    v = dpp_wave_sum(v);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < JOIN / 64; ++i) sum += lds[i];
    return sum;
}

// f(chunk, channel of the group, its two sums) of the parts of a group
template <class F> __device__ __forceinline__ void for_parts(const WideCall& f, int64_t image, int first, F of) {
    const int channels = f.n.channels, D = channels / f.n.groups;
    const float* parts = f.parts + image * f.chunks * 2 * channels + first;
    for (int j = 0; j < f.chunks; ++j, parts += 2 * (int64_t)channels) {
#pragma unroll 8
        for (int d = threadIdx.x; d < D; d += JOIN) of(j, d, parts[d], (parts + channels)[d]);
    }
}

// mean and r of a group: a workgroup per group
__global__ void __launch_bounds__(JOIN) norm_wide_join_kernel(WideCall f) {
    __shared__ float lds[JOIN / 64];
    const NormCall& c = f.n;
    const int D = c.channels / c.groups;
    const float n = (float)c.positions * (float)D, whole = (float)f.rows, last = (float)(c.positions - (f.chunks - 1) * f.rows);
    for (int64_t g = blockIdx.x; g < c.sets * c.images * c.groups; g += gridDim.x) {
        const int64_t image = g / c.groups;
        const int first = (int)(g - image * c.groups) * D;
        float mean = 0.f, var = 0.f;
        if (f.chunks) {
            double sum = 0.;
            for_parts(f, image, first, [&](int j, int, float m, float) { sum += (j < f.chunks - 1 ? whole : last) * m; });
            mean = block_sum((float)sum, lds) / n;
            sum = 0.;
            for_parts(f, image, first, [&](int j, int, float m, float q) { sum += q + (j < f.chunks - 1 ? whole : last) * (m - mean) * (m - mean); });
            var = block_sum((float)sum, lds) / n;
        }
        if (threadIdx.x == 0) {
            const float r = 1.f / sqrtf(var + c.eps);
            f.mean[g] = mean;
            f.rstd[g] = r;
            if (c.mean) { c.mean[g] = mean; c.rstd[g] = r; }
        }
    }
}

// A and B of a group: a workgroup per group
__global__ void __launch_bounds__(JOIN) norm_wide_group_kernel(WideCall f, float* group_sums) {
    __shared__ float lds[JOIN / 64];
    const NormCall& c = f.n;
    const int D = c.channels / c.groups;
    const float n = (float)c.positions * (float)D;
    for (int64_t g = blockIdx.x; g < c.sets * c.images * c.groups; g += gridDim.x) {
        const int64_t image = g / c.groups;
        const int first = (int)(g - image * c.groups) * D;
        const float* w = c.weight ? c.weight + (uint32_t)image / (uint32_t)c.images * c.weight_stride + first : nullptr;
        double a = 0., b = 0.;
        for_parts(f, image, first, [&](int, int d, float dz, float dzx) {
            const float wd = w ? w[d] : 1.f;
            a += wd * dz;
            b += wd * dzx;
        });
        const float A = block_sum((float)a, lds) / n, B = block_sum((float)b, lds) / n;
        if (threadIdx.x == 0) { group_sums[2 * g] = A; group_sums[2 * g + 1] = B; }
    }
}

template <class E, bool SILU>
__global__ void __launch_bounds__(T) norm_wide_apply_kernel(WideCall f) {
    const NormCall& c = f.n;
    for (int64_t image = blockIdx.z; image < f.n.sets * f.n.images; image += gridDim.z) {
        const WidePlace l(f, image);
        if (!l.on) continue;
        const E* x = l.at<const E>(c.x, c.xs);
        E* y = l.at<E>(c.out, c.outs);
        const float mean = f.mean[l.image * c.groups + l.group], rstd = f.rstd[l.image * c.groups + l.group];
        const float w = c.weight ? c.weight[l.set * c.weight_stride + l.ch] : 1.f, b = c.bias ? c.bias[l.set * c.bias_stride + l.ch] : 0.f;
        const uint64_t number = l.number(c);
        for_rows(l.rows, [&](int64_t s, auto some) {
            constexpr int K = some.value;
            float v[K];
#pragma unroll
            for (int i = 0; i < K; ++i) v[i] = to_float(x[(s + i) * c.xs.row]);
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const float z = (v[i] - mean) * rstd * w + b;
                float a = SILU ? SILU_BACK * activate<true>(SILU_SCALE * z, 0.f) : activate<false>(z, c.floor);
                if (c.drop.threshold) a = drop_keeps(c.drop, number + (uint64_t)(s + i) * c.channels) ? a * c.drop.scale : 0.f;
                y[(s + i) * c.outs.row] = from_float<E>(a);
            }
        });
    }
}

// f(position in the chunk, dz, x - m) of a lane's channel, and after() behind every ROWS of them, or one
template <class E, bool SILU, class F, class After>
__device__ __forceinline__ void for_gradients(const NormCall& c, const WidePlace& l, float w, float mean, float rstd, F f, After after) {
    const E* x = l.at<const E>(c.x, c.xs);
    const E* dy = l.at<const E>(c.dy, c.dys);
    const float b = c.bias ? c.bias[l.set * c.bias_stride + l.ch] : 0.f;
    const uint64_t number = l.number(c);
    for_rows(l.rows, [&](int64_t s, auto some) {
        constexpr int K = some.value;
        float v[K], g[K];
#pragma unroll
        for (int i = 0; i < K; ++i) { v[i] = to_float(x[(s + i) * c.xs.row]); g[i] = to_float(dy[(s + i) * c.dys.row]); }
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const float d = v[i] - mean, z = d * rstd * w + b;
            if (c.drop.threshold) g[i] = drop_keeps(c.drop, number + (uint64_t)(s + i) * c.channels) ? g[i] * c.drop.scale : 0.f;
            f(s + i, through_slope<SILU>(g[i], SILU ? SILU_SCALE * z : z, c.floor), d);
        }
        after();
    });
}

template <class E, bool SILU>
__global__ void __launch_bounds__(T) norm_wide_sums_kernel(WideCall f) {
    const NormCall& c = f.n;
    for (int64_t image = blockIdx.z; image < f.n.sets * f.n.images; image += gridDim.z) {
        const WidePlace l(f, image);
        if (!l.on) continue;
        const float mean = c.mean[l.image * c.groups + l.group], rstd = c.rstd[l.image * c.groups + l.group];
        double a = 0., b = 0.;
        float some = 0.f, some_d = 0.f;
        for_gradients<E, SILU>(c, l, c.weight ? c.weight[l.set * c.weight_stride + l.ch] : 1.f, mean, rstd,
                               [&](int64_t, float dz, float d) { some += dz; some_d += dz * d; }, [&] { a += some; b += some_d; some = some_d = 0.f; });
        float* to = l.parts(f);
        to[0] = (float)a;
        to[c.channels] = (float)b * rstd;
    }
}

template <class E, bool SILU>
__global__ void __launch_bounds__(T) norm_wide_dx_kernel(WideCall f) {
    const NormCall& c = f.n;
    for (int64_t image = blockIdx.z; image < f.n.sets * f.n.images; image += gridDim.z) {
        const WidePlace l(f, image);
        if (!l.on) continue;
        const int64_t g = l.image * c.groups + l.group;
        const float w = c.weight ? c.weight[l.set * c.weight_stride + l.ch] : 1.f, mean = c.mean[g], rstd = c.rstd[g], A = f.group_sums[2 * g], B = f.group_sums[2 * g + 1];
        E* dx = l.at<E>(c.out, c.outs);
        for_gradients<E, SILU>(c, l, w, mean, rstd,
                               [&](int64_t s, float dz, float d) { dx[s * c.outs.row] = from_float<E>(rstd * (w * dz - A - d * rstd * B)); }, [] {});
    }
}

// channels, chunks, images of a launch: some thousand workgroups, and images one after the other where there are more (1024 vectors of 16384
// channels, backward: 191 us, a workgroup for every one of them 281)
dim3 wide_grid(const NormCall& c, int chunks) {
    const int64_t blocks = (c.channels + T - 1) / T, most = std::max<int64_t>(1, MOST_GROUPS / (blocks * chunks));
    return dim3((unsigned)blocks, (unsigned)chunks, (unsigned)std::min({c.sets * c.images, most, (int64_t)65535}));
}

size_t wide_workspace(const NormCall& c) {
    if (!c.positions) return 0;
    return (size_t)c.sets * c.images * (2 * (size_t)chunks_of(c).count * c.channels + 2 * (size_t)c.groups) * sizeof(float);
}

template <class E>
hipError_t wide_forward(const NormCall& c, float* workspace, hipStream_t st) {
    const Chunks k = chunks_of(c);
    const int64_t images = c.sets * c.images, groups = images * c.groups;
    WideCall f = {c, k.rows, k.count, workspace, workspace + images * k.count * 2 * c.channels, nullptr, nullptr};
    f.rstd = f.mean + groups;
    if (!c.positions) {                              // (statistics of nothing, for whom they concern)
        if (!c.mean) return hipSuccess;
        f.mean = c.mean;
        f.rstd = c.rstd;
    }
    const dim3 grid = wide_grid(c, std::max(1, k.count)), block(T);
    if (k.count) norm_wide_moments_kernel<E><<<grid, block, 0, st>>>(f);
    norm_wide_join_kernel<<<loop_grid(groups), dim3(JOIN), 0, st>>>(f);
    if (k.count) {
        if (c.silu) norm_wide_apply_kernel<E, true><<<grid, block, 0, st>>>(f);
        else norm_wide_apply_kernel<E, false><<<grid, block, 0, st>>>(f);
    }
    return hipGetLastError();
}

template <class E, bool SILU>
hipError_t wide_backward(const NormCall& c, float* workspace, hipStream_t st) {
    const Chunks k = chunks_of(c);
    const int64_t images = c.sets * c.images, groups = images * c.groups;
    float* group_sums = workspace + images * k.count * 2 * c.channels;
    const WideCall f = {c, k.rows, k.count, workspace, nullptr, nullptr, group_sums};
    BackwardCall b = {};
    b.n = c;
    b.parts = workspace;
    b.chunks = k.count;
    const dim3 grid = wide_grid(c, std::max(1, k.count)), block(T);
    if (groups && k.count) {
        norm_wide_sums_kernel<E, SILU><<<grid, block, 0, st>>>(f);
        norm_wide_group_kernel<<<loop_grid(groups), dim3(JOIN), 0, st>>>(f, group_sums);
        norm_wide_dx_kernel<E, SILU><<<grid, block, 0, st>>>(f);
    }
    const int64_t params = param_blocks(b);
    if (params) norm_param_kernel<1024><<<loop_grid(params), dim3(1024), 2 * 1024 * sizeof(float), st>>>(b);
    return hipGetLastError();
}

hipError_t check(size_t want, const void* workspace, size_t bytes) {
    if (want > bytes) return hipErrorOutOfMemory;
    return want && (!workspace || ((uintptr_t)workspace & 15)) ? hipErrorInvalidValue : hipSuccess;
}

template <class E>
hipError_t backward(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    if (!c.sets) return hipSuccess;
    NormTiles t;
    const bool tiled = c.images && c.positions && call_tiles(c, true, &t);
    const hipError_t e = check(tiled ? norm_workspace(c, t, true) : wide_workspace(c), workspace, bytes);
    if (e != hipSuccess) return e;
    if (tiled) return tiled_backward<E>(c, t, workspace, st);
    return c.silu ? wide_backward<E, true>(c, (float*)workspace, st) : wide_backward<E, false>(c, (float*)workspace, st);
}

template <class E>
hipError_t forward(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    if (!(c.sets * c.images)) return hipSuccess;
    NormTiles t;
    const bool tiled = c.positions && call_tiles(c, false, &t);
    const hipError_t e = check(tiled ? norm_workspace(c, t, false) : wide_workspace(c), workspace, bytes);
    if (e != hipSuccess) return e;
    return tiled ? tiled_forward<E>(c, t, workspace, st) : wide_forward<E>(c, (float*)workspace, st);
}

}  // namespace

size_t norm_workspace(const NormCall& c, bool backward) {
    NormTiles t;
    size_t most = 0;
    for (const bool contiguous : {true, false}) {
        const bool tiled = c.sets && c.images && c.positions && norm_tiles(c, contiguous, backward, &t);
        most = std::max(most, tiled ? norm_workspace(c, t, backward) : wide_workspace(c));
        if (c.channels % (c.dtype == KAVG_BF16 ? 8 : 4) == 0) break;       // (it makes no difference)
    }
    return most;
}

hipError_t launch_group_norm(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    return c.dtype == KAVG_BF16 ? forward<__bf16>(c, workspace, bytes, st) : forward<float>(c, workspace, bytes, st);
}

hipError_t launch_group_norm_backward(const NormCall& c, void* workspace, size_t bytes, hipStream_t st) {
    return c.dtype == KAVG_BF16 ? backward<__bf16>(c, workspace, bytes, st) : backward<float>(c, workspace, bytes, st);
}

}  // namespace kavg
