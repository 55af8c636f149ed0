// Launches of the tiled backward pass, and the sums behind its tiles.
#include "norm_backward.h"

namespace kavg {

namespace {

constexpr size_t LDS_PLAIN = 64 * 1024;      // more than that has to be asked for

int64_t extent_of(const NormCall& c, const Strides& s) {
    return (c.sets - 1) * s.set + (c.images - 1) * s.image + (c.positions - 1) * s.row + c.channels;
}

// A and B of a group from the sums of its image's chunks: a workgroup per group
__global__ void __launch_bounds__(256) norm_group_kernel(const float* parts, const float* weight, int64_t weight_stride, int64_t images, int chunks,
                                                         int channels, int groups, float n, float* group_sums) {
    __shared__ float lds[8];
    const int64_t image = blockIdx.x / groups;
    const int D = channels / groups, first = (int)(blockIdx.x % groups) * D;
    const float* p = parts + image * chunks * 2 * channels + first;
    const float* w = weight ? weight + image / images * weight_stride + first : nullptr;
    float a = 0.f, b = 0.f;
    for (int j = threadIdx.x, r = j / D, i = j - r * D; r < chunks; ) {
        const float wi = w ? w[i] : 1.f;
        a += wi * p[(int64_t)r * 2 * channels + i];
        b += wi * p[(int64_t)r * 2 * channels + channels + i];
        i += 256;
        if (i >= D) { const int over = i / D; r += over; i -= over * D; }
    }
    a = team_sum(a, 64);
    b = team_sum(b, 64);
    if (threadIdx.x % 64 == 0) { lds[threadIdx.x / 64] = a; lds[4 + threadIdx.x / 64] = b; }
    __syncthreads();
    if (threadIdx.x < 2) {
        const float* q = lds + 4 * threadIdx.x;
        group_sums[2 * (int64_t)blockIdx.x + threadIdx.x] = ((q[0] + q[1]) + (q[2] + q[3])) / n;
    }
}

// dweight and dbias: a learner's sums over its images and their chunks.  A workgroup: `wide` channels (a power of two), the rows dealt
// out to 1024 / wide lanes each, then these in order.
__global__ void __launch_bounds__(1024) norm_param_kernel(const float* parts, int64_t rows, int channels, int wide, int blocks, float* dweight,
                                                          int64_t dweight_stride, float* dbias, int64_t dbias_stride) {
    __shared__ float lds[2][1024];
    const int64_t set = blockIdx.x / blocks;
    const int ch = (int)(blockIdx.x % blocks) * wide + threadIdx.x % wide, share = threadIdx.x / wide, shares = 1024 / wide;
    float a = 0.f, b = 0.f;
    if (ch < channels) {
        const float* p = parts + set * rows * 2 * channels + ch;
#pragma unroll 8
        for (int64_t r = share; r < rows; r += shares) { a += p[r * 2 * channels]; b += p[r * 2 * channels + channels]; }
    }
    lds[0][threadIdx.x] = a;
    lds[1][threadIdx.x] = b;
    __syncthreads();
    // halves onto halves
    for (int s = 512; s >= wide; s /= 2) {
        if ((int)threadIdx.x < s) { lds[0][threadIdx.x] += lds[0][threadIdx.x + s]; lds[1][threadIdx.x] += lds[1][threadIdx.x + s]; }
        __syncthreads();
    }
    if (share == 0 && ch < channels) {
        if (dbias) dbias[set * dbias_stride + ch] = lds[0][threadIdx.x];
        if (dweight) dweight[set * dweight_stride + ch] = lds[1][threadIdx.x];
    }
}

template <class E, int V, int NV, bool FLAT, bool WHOLE_PACK, int MODE>
hipError_t start(const BackwardCall& f, hipStream_t st) {
    const auto kernel = norm_backward_kernel<E, V, NV, FLAT, WHOLE_PACK, MODE>;
    const Tile& t = f.t;
    const int64_t images = f.n.sets * f.n.images, grid = (images + t.units - 1) / t.units * t.blocks * t.chunks;
    if (grid >= (int64_t)1 << 31) return hipErrorInvalidConfiguration;
    const size_t lds = MODE == TILE_APPLY ? 0 : t.lds;
    if (lds > LDS_PLAIN) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)grid), dim3(t.threads), lds, st>>>(f);
    return hipGetLastError();
}

template <class E, int V, int NV, int MODE>
hipError_t of_layout(const BackwardCall& f, hipStream_t st) {
    if constexpr (V == 1) return start<E, 1, NV, false, true, MODE>(f, st);
    else if (f.t.flat) return start<E, V, NV, true, false, MODE>(f, st);
    else return f.t.whole_pack ? start<E, V, NV, false, true, MODE>(f, st) : start<E, V, NV, false, false, MODE>(f, st);
}

template <class E, int V, int MODE>
hipError_t of_packs(const BackwardCall& f, hipStream_t st) {
    if (MODE != TILE_WHOLE) return of_layout<E, V, BACKWARD_PACKS, MODE>(f, st);
    switch (f.t.nv) {
        case 1: return of_layout<E, V, 1, TILE_WHOLE>(f, st);
        case 2: return of_layout<E, V, 2, TILE_WHOLE>(f, st);
        default: return of_layout<E, V, BACKWARD_PACKS, TILE_WHOLE>(f, st);
    }
}

template <class E, int V>
hipError_t backward(BackwardCall& f, float* workspace, hipStream_t st) {
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const int64_t images = c.sets * c.images, groups = images * c.groups;
    const bool params = c.dweight || c.dbias;
    f.parts = params || t.chunks > 1 ? workspace : nullptr;
    hipError_t e;
    if (t.chunks == 1) {
        e = of_packs<E, V, TILE_WHOLE>(f, st);
        if (e != hipSuccess) return e;
    } else {
        float* group_sums = workspace + images * t.chunks * 2 * c.channels;
        f.group_sums = group_sums;
        e = of_packs<E, V, TILE_SUMS>(f, st);
        if (e != hipSuccess) return e;
        norm_group_kernel<<<dim3((unsigned)groups), dim3(256), 0, st>>>(f.parts, c.weight, c.weight_stride, c.images, t.chunks, c.channels, c.groups,
                                                                         (float)c.positions * (float)(c.channels / c.groups), group_sums);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        e = of_packs<E, V, TILE_APPLY>(f, st);
        if (e != hipSuccess) return e;
    }
    if (!params) return hipSuccess;
    int wide = 64;
    while (wide > 1 && wide / 2 >= c.channels) wide /= 2;
    const int blocks = (c.channels + wide - 1) / wide;
    norm_param_kernel<<<dim3((unsigned)(c.sets * blocks)), dim3(1024), 0, st>>>(f.parts, c.images * t.chunks, c.channels, wide, blocks, c.dweight,
                                                                                 c.dweight_stride, c.dbias, c.dbias_stride);
    return hipGetLastError();
}

}  // namespace

template <class E> hipError_t tiled_backward(const NormCall& c, const Tile& t, void* workspace, hipStream_t st) {
    BackwardCall f = {c, t, extent_of(c, c.xs), extent_of(c, c.dys), nullptr, nullptr};
    return t.vec == 1 ? backward<E, 1>(f, (float*)workspace, st) : backward<E, 16 / (int)sizeof(E)>(f, (float*)workspace, st);
}
template hipError_t tiled_backward<float>(const NormCall&, const Tile&, void*, hipStream_t);
template hipError_t tiled_backward<__bf16>(const NormCall&, const Tile&, void*, hipStream_t);

}  // namespace kavg
