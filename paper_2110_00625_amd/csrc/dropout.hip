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

constexpr int T = 256;

// U packs of V elements (16 bytes) per lane, T packs apart; pack i of the tensor lies in row i / per_row.  A row's last pack, if V does
// not divide its length, is the last V elements, of which the pack before has had `skip`: they are read for nothing and not written
// (in place they may have changed by then).  No load stands behind a branch: a lane with nothing to do reads the last pack.
template <class E, int U, bool ROWS, bool ALIGNED, bool RESIDUAL>
__device__ __forceinline__ void packs_of_lane(const DropCall& c, uint64_t first, uint64_t per_row, Divisor by_row) {
    constexpr int V = 16 / sizeof(E);
    typedef typename Pack<E, V>::type pack;
    const uint64_t total = per_row * c.rows;
    // (ROWS: per_row < 2^28, so that what is divided stays below 2^30)
    const uint64_t row0 = ROWS ? first / per_row : 0;
    const uint32_t pack0 = (uint32_t)(first - row0 * per_row);
    uint64_t row[U], col[U];
    int skip[U];                                            // V: nothing to do
    pack xv[U], rv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint32_t i = u * T + threadIdx.x;
        const bool none = first + i >= total;
        if (none) i = (uint32_t)(total - 1 - first);
        row[u] = 0;
        if (ROWS) {
            const uint32_t r = divide(pack0 + i, by_row);
            row[u] = row0 + r;
            col[u] = (uint64_t)(pack0 + i - r * (uint32_t)per_row) * V;
        } else col[u] = (first + i) * V;
        skip[u] = 0;
        if (!ALIGNED || ROWS) {
            const int64_t over = (int64_t)col[u] + V - c.cols;
            if (over > 0) { col[u] -= over; skip[u] = (int)over; }
        }
        if (none) skip[u] = V;
        xv[u] = pack_load<E, V>((const E*)c.x + row[u] * c.x_stride + col[u]);
        if (RESIDUAL) rv[u] = pack_load<E, V>((const E*)c.residual + row[u] * c.residual_stride + col[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (c.drop.threshold) drop_pack<E, V, ALIGNED>(c.drop, DropPlace(c.drop, row[u] * c.cols + col[u]), xv[u]);
        pack o;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float v = to_float(xv[u][i]) * c.drop.scale;
            o[i] = from_float<E>(RESIDUAL ? v + to_float(rv[u][i]) : v);
        }
        E* y = (E*)c.y + row[u] * c.y_stride + col[u];
        if (skip[u] == 0) pack_store<E, V>(y, o);
        else {
#pragma unroll
            for (int i = 1; i < V; ++i) if (i >= skip[u]) y[i] = o[i];
        }
    }
}

template <class E, int U, bool ROWS, bool ALIGNED, bool RESIDUAL>
__global__ void __launch_bounds__(T) dropout_kernel(DropCall c, uint64_t per_row, Divisor by_row) {
    constexpr int V = 16 / sizeof(E);
    const uint64_t first = (uint64_t)blockIdx.x * (U * T);
    if (ROWS) packs_of_lane<E, U, true, ALIGNED, RESIDUAL>(c, first, per_row, by_row);
    else if (first + U * T <= (uint64_t)c.cols / V) packs_of_lane<E, U, false, true, RESIDUAL>(c, first, per_row, by_row);
    else packs_of_lane<E, U, false, false, RESIDUAL>(c, first, per_row, by_row);     // the end of the tensor
}

// rows of fewer than V elements: an element per lane
template <class E>
__global__ void __launch_bounds__(T) dropout_short_kernel(DropCall c) {
    const uint64_t e = (uint64_t)blockIdx.x * T + threadIdx.x;
    if (e >= (uint64_t)c.rows * c.cols) return;
    const uint64_t r = e / c.cols, k = e - r * c.cols;
    float v = to_float(((const E*)c.x)[r * c.x_stride + k]);
    if (c.drop.threshold) v = drop_keeps(c.drop, e) ? v * c.drop.scale : 0.f;
    if (c.residual) v += to_float(((const E*)c.residual)[r * c.residual_stride + k]);
    ((E*)c.y)[r * c.y_stride + k] = from_float<E>(v);
}

template <class E, int U, bool ROWS, bool ALIGNED>
void start(const DropCall& c, uint64_t per_row, hipStream_t st) {
    const Divisor by_row = ROWS ? divisor((uint32_t)per_row) : Divisor{0, 0};
    const dim3 grid((unsigned)((per_row * c.rows + U * T - 1) / (U * T)));
    if (c.residual) dropout_kernel<E, U, ROWS, ALIGNED, true><<<grid, dim3(T), 0, st>>>(c, per_row, by_row);
    else dropout_kernel<E, U, ROWS, ALIGNED, false><<<grid, dim3(T), 0, st>>>(c, per_row, by_row);
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
    if (c.cols < V) dropout_short_kernel<E><<<dim3((unsigned)((c.rows * c.cols + T - 1) / T)), dim3(T), 0, st>>>(c);
    else if (c.rows > 1) {
        if (c.cols % 4 == 0) start<E, 1, true, true>(c, per_row, st);
        else start<E, 1, true, false>(c, per_row, st);
    } else if (per_row >= 4 * T * 1024) start<E, 4, false, true>(c, per_row, st);
    else start<E, 1, false, true>(c, per_row, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropCall& c, hipStream_t st) {
    if (!c.rows) return hipSuccess;
    return c.dtype == KAVG_BF16 ? launch<__bf16>(c, st) : launch<float>(c, st);
}

}  // namespace kavg
