// Dropout from a counter-based generator: y = keep ? x / (1 - p) : 0, plus a residual.  The mask is a function of the element's number
// (counter_stream.h), so the backward pass draws it again and nothing is stored.  An element is read and written once, and a draw of
// 64 bits, some thirty instructions, serves four of them: bound by memory.  A pack per lane (four per lane, their loads in flight together, were
// the same within 4 % either way).  67M elements in bf16 40 us, 6.6 TB/s, part of it in the 256 MB cache behind the L2, 47 us out of memory; 2048 rows
// of 4096 in bf16 with a residual 9.0 us, 5.6 TB/s; 4999 rows of 1001 in fp32 7.9 us, 5.1 TB/s; 192 rows of 256 2.4 us of a call
// of 7.8, which is the host's time.
#include "layers.h"
#include <algorithm>
#include <cmath>

namespace kavg {

DropRule drop_rule(double drop, uint64_t seed, uint64_t site) {
    const uint32_t t = (uint32_t)std::floor(drop * 65536 + 0.5);
    return {seed + (1 + (site << 40)) * SPLITMIX_GAMMA, t, t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.f};
}

namespace {

constexpr int T = 256;

// A pack of V elements (16 bytes) per lane; pack i of the tensor lies in row i / per_row.  A row's last pack, if V does not divide its
// length, is the last V elements, of which the pack before has had `skip`: they are read for nothing and not written (in place they may
// have changed by then).  No load stands behind a branch: a lane with nothing to do reads the last pack.
template <class E, bool ROWS, bool ALIGNED, bool RESIDUAL>
__device__ __forceinline__ void pack_of_lane(const DropCall& c, uint64_t first, uint64_t per_row, Divisor by_row) {
    constexpr int V = 16 / sizeof(E);
    typedef typename Pack<E, V>::type pack;
    const uint64_t total = per_row * c.rows;
    uint32_t i = threadIdx.x;
    const bool none = first + i >= total;
    if (none) i = (uint32_t)(total - 1 - first);
    uint64_t row = 0, col;
    if (ROWS) {                                             // (per_row < 2^28, so that what is divided stays below 2^30)
        const uint64_t row0 = first / per_row;
        const uint32_t pack0 = (uint32_t)(first - row0 * per_row), r = divide(pack0 + i, by_row);
        row = row0 + r;
        col = (uint64_t)(pack0 + i - r * (uint32_t)per_row) * V;
    } else col = (first + i) * V;
    int skip = 0;                                           // V: nothing to do
    if (!ALIGNED || ROWS) {
        const int64_t over = (int64_t)col + V - c.cols;
        if (over > 0) { col -= over; skip = (int)over; }
    }
    if (none) skip = V;
    pack xv = pack_load<E, V>((const E*)c.x + row * c.x_stride + col), rv;
    if (RESIDUAL) rv = pack_load<E, V>((const E*)c.residual + row * c.residual_stride + col);
    if (c.drop.threshold) drop_pack<E, V, ALIGNED>(c.drop, DropPlace(c.drop, row * c.cols + col), xv);
    pack o;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const float v = to_float(xv[k]) * c.drop.scale;
        o[k] = from_float<E>(RESIDUAL ? v + to_float(rv[k]) : v);
    }
    E* y = (E*)c.y + row * c.y_stride + col;
    if (skip == 0) pack_store<E, V>(y, o);
    else {
#pragma unroll
        for (int k = 1; k < V; ++k) if (k >= skip) y[k] = o[k];
    }
}

template <class E, bool ROWS, bool ALIGNED, bool RESIDUAL>
__global__ void __launch_bounds__(T) dropout_kernel(DropCall c, uint64_t per_row, Divisor by_row) {
    constexpr int V = 16 / sizeof(E);
    for (uint64_t first = (uint64_t)blockIdx.x * T; first < per_row * c.rows; first += (uint64_t)gridDim.x * T) {
        if (ROWS) pack_of_lane<E, true, ALIGNED, RESIDUAL>(c, first, per_row, by_row);
        else if (first + T <= (uint64_t)c.cols / V) pack_of_lane<E, false, true, RESIDUAL>(c, first, per_row, by_row);
        else pack_of_lane<E, false, false, RESIDUAL>(c, first, per_row, by_row);     // the end of the tensor
    }
}

// rows of fewer than V elements: an element per lane
template <class E>
__global__ void __launch_bounds__(T) dropout_short_kernel(DropCall c) {
    for (uint64_t e = (uint64_t)blockIdx.x * T + threadIdx.x; e < (uint64_t)c.rows * c.cols; e += (uint64_t)gridDim.x * T) {
        const uint64_t r = e / c.cols, k = e - r * c.cols;
        float v = to_float(((const E*)c.x)[r * c.x_stride + k]);
        if (c.drop.threshold) v = drop_keeps(c.drop, e) ? v * c.drop.scale : 0.f;
        if (c.residual) v += to_float(((const E*)c.residual)[r * c.residual_stride + k]);
        ((E*)c.y)[r * c.y_stride + k] = from_float<E>(v);
    }
}

// a lane for each of n packs, but fewer than 2^32 (what a launch takes): from there on a lane takes several, 2^22 workgroups apart
dim3 grid_of(uint64_t n) { return dim3((unsigned)std::min<uint64_t>((n + T - 1) / T, 1 << 22)); }

template <class E, bool ROWS, bool ALIGNED>
void start(const DropCall& c, uint64_t per_row, hipStream_t st) {
    const Divisor by_row = ROWS ? divisor((uint32_t)per_row) : Divisor{0, 0};
    const dim3 grid = grid_of(per_row * c.rows);
    if (c.residual) dropout_kernel<E, ROWS, ALIGNED, true><<<grid, dim3(T), 0, st>>>(c, per_row, by_row);
    else dropout_kernel<E, ROWS, ALIGNED, false><<<grid, dim3(T), 0, st>>>(c, per_row, by_row);
}

template <class E>
hipError_t launch(const DropCall& call, hipStream_t st) {
    constexpr int V = 16 / sizeof(E);
    DropCall c = call;
    if (c.x_stride == c.cols && c.y_stride == c.cols && (!c.residual || c.residual_stride == c.cols)) {
        c.cols *= c.rows;                                   // one row
        c.rows = 1;
    }
    const uint64_t per_row = (c.cols + V - 1) / V;
    if (c.cols < V) dropout_short_kernel<E><<<grid_of((uint64_t)c.rows * c.cols), dim3(T), 0, st>>>(c);
    else if (c.rows == 1) start<E, false, true>(c, per_row, st);
    else if (c.cols % 4 == 0) start<E, true, true>(c, per_row, st);
    else start<E, true, false>(c, per_row, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropCall& c, hipStream_t st) {
    if (!c.rows) return hipSuccess;
    return c.dtype == KAVG_BF16 ? launch<__bf16>(c, st) : launch<float>(c, st);
}

}  // namespace kavg
