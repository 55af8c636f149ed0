// Launches of the tiled forward pass.
#include "norm_forward.h"

namespace kavg {

namespace {

constexpr size_t LDS_PLAIN = 64 * 1024;      // more than that has to be asked for

int64_t extent_of(const NormCall& c, const Strides& s) {
    return (c.sets - 1) * s.set + (c.images - 1) * s.image + (c.positions - 1) * s.row + c.channels;
}

template <class E, int V, int NV, bool FLAT, bool WHOLE_PACK, int MODE>
hipError_t start(const ForwardCall& f, hipStream_t st) {
    const auto kernel = norm_forward_kernel<E, V, NV, FLAT, WHOLE_PACK, MODE>;
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
hipError_t of_layout(const ForwardCall& f, hipStream_t st) {
    if constexpr (V == 1) return start<E, 1, NV, false, true, MODE>(f, st);
    else if (f.t.flat) return start<E, V, (NV < FLAT_PACKS ? NV : FLAT_PACKS), true, false, MODE>(f, st);
    else return f.t.whole_pack ? start<E, V, NV, false, true, MODE>(f, st) : start<E, V, NV, false, false, MODE>(f, st);
}

template <class E, int V, int MODE>
hipError_t of_packs(const ForwardCall& f, hipStream_t st) {
    if (MODE != TILE_WHOLE) return of_layout<E, V, 16, MODE>(f, st);
    switch (f.t.nv) {
        case 1: return of_layout<E, V, 1, TILE_WHOLE>(f, st);
        case 2: return of_layout<E, V, 2, TILE_WHOLE>(f, st);
        case 4: return of_layout<E, V, 4, TILE_WHOLE>(f, st);
        case 8: return of_layout<E, V, 8, TILE_WHOLE>(f, st);
        default: return of_layout<E, V, 16, TILE_WHOLE>(f, st);
    }
}

template <class E, int V>
hipError_t forward(ForwardCall& f, void* workspace, hipStream_t st) {
    if (f.t.chunks == 1) return of_packs<E, V, TILE_WHOLE>(f, st);
    const NormCall& c = f.n;
    const int64_t groups = c.sets * c.images * c.groups;
    f.parts = (float*)workspace;
    float* mean = f.parts + 2 * groups * f.t.chunks;
    float* rstd = mean + groups;
    f.mean = mean;
    f.rstd = rstd;
    hipError_t e = of_packs<E, V, TILE_SUMS>(f, st);
    if (e != hipSuccess) return e;
    // values of a group in a whole chunk and in the last one
    const int64_t rows = f.t.flat ? (int64_t)f.t.cols * f.t.vec / c.channels : f.t.lane_rows, whole = f.t.nv * rows;
    const float per = (float)(c.channels / c.groups);
    norm_join_kernel<256><<<dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, st>>>(
        f.parts, f.t.chunks, groups, (float)whole * per, (float)(c.positions - whole * (f.t.chunks - 1)) * per, c.eps, mean, rstd, c.mean, c.rstd);
    e = hipGetLastError();
    return e == hipSuccess ? of_packs<E, V, TILE_APPLY>(f, st) : e;
}

}  // namespace

template <class E> hipError_t tiled_forward(const NormCall& c, const Tile& t, void* workspace, hipStream_t st) {
    ForwardCall f = {c, t, extent_of(c, c.xs), nullptr, nullptr, nullptr};
    return t.vec == 1 ? forward<E, 1>(f, workspace, st) : forward<E, 16 / (int)sizeof(E)>(f, workspace, st);
}
template hipError_t tiled_forward<float>(const NormCall&, const Tile&, void*, hipStream_t);
template hipError_t tiled_forward<__bf16>(const NormCall&, const Tile&, void*, hipStream_t);

}  // namespace kavg
