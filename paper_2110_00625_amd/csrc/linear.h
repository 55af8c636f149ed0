// Launch interface of the products (kavg_linear, kavg_linear_backward) and what their kernels share.  The boundary (learner_api.hip)
// has checked every argument.
//
// All three products of a layer are  O[r][c] = sum_k R(r,k) C(c,k)  per learner:
//   forward          r = row,     c = output, k = input     R = x,           C = W
//   data gradient    r = row,     c = input,  k = output    R = dz,          C = W turned
//   weight gradient  r = output,  c = input,  k = row       R = dz turned,   C = x turned
// (of weights that lie as [inputs][outputs] the other way round: C = W turned, C = W, and R = x turned, C = dz turned).
#pragma once
#include "kavg_internal.h"
#include "layers.h"

namespace kavg {

// Element (x, k) of a learner's matrix: base[set * set_stride + x * stride + k], or of a turned one base[.. + k * stride + x].
struct Matrix { const void* base; int64_t set_stride, stride; };

// What becomes of a product's values v(r, c).  Pointers that are null are left out, in this order:
//   v += bias[c];  kept[r][c] = v;  v = act(v);  v *= slope(before[r][c]);  v += residual[r][c];  out[r][c] = v
struct Finish {
    const float* bias; int64_t bias_set;
    void* kept; int64_t kept_set, kept_row;
    bool silu; float floor;                      // act: see layers.h
    const void* before; int64_t before_set, before_row;
    bool slope_silu;
    const void* residual; int64_t residual_set, residual_row;
    void* out; int64_t out_set, out_row;         // of the operands' type, of a weight gradient fp32
};

struct ProductCall {
    int dtype;
    int64_t sets;
    int nR, nC, nK;
    Matrix R, C;
    bool r_turned, c_turned;                     // (r_turned: a weight gradient, c_turned too)
    Finish finish;
    // sums over k of R (side 1) or C (side 2), of a weight gradient: those of dz are the bias's gradient
    int side; float* sums; int64_t sums_set;
};

// How a product is cut: the tile (linear_tile.h), and between how many workgroups a tile's contraction is split.  Their partial results, [split]
// [set][r][c] in fp32 with rows of `pitch`, and sums lie in the workspace; the launch that joins them finishes the values.
struct Plan {
    int tile, splits, pitch;
    size_t bytes;                                // of workspace
};
enum Turned { NONE_TURNED, C_TURNED, BOTH_TURNED };        // the last: a weight gradient
Plan product_plan(int dtype, int64_t sets, int nR, int nC, int nK, Turned turned);
// hipErrorOutOfMemory, hipErrorInvalidValue: a workspace too small, misaligned or not there, before anything is launched
hipError_t launch_product(const ProductCall& c, void* workspace, size_t bytes, hipStream_t st);
hipError_t check_product(const ProductCall& c, const void* workspace, size_t bytes);       // the same, without the launch

#if defined(__HIPCC__)
template <class E, int V> __device__ __forceinline__ void load_some(const E* p, int n, float (&v)[V]) {
    if (n >= V) {
#pragma unroll
        for (int i = 0; i < V; i += 16 / sizeof(E) < V ? 16 / sizeof(E) : V) {
            constexpr int W = 16 / sizeof(E) < V ? 16 / sizeof(E) : V;
            const auto q = pack_load<E, W>(p + i);
#pragma unroll
            for (int k = 0; k < W; ++k) v[i + k] = to_float(q[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = k < n ? to_float(p[k]) : 0.f;
    }
}
template <class E, int V> __device__ __forceinline__ void store_some(E* p, int n, const float (&v)[V]) {
    if (n >= V) {
        constexpr int W = 16 / sizeof(E) < V ? 16 / sizeof(E) : V;
#pragma unroll
        for (int i = 0; i < V; i += W) {
            typename Pack<E, W>::type q;
#pragma unroll
            for (int k = 0; k < W; ++k) q[k] = from_float<E>(v[i + k]);
            pack_store<E, W>(p + i, q);
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) if (k < n) p[k] = from_float<E>(v[k]);
    }
}

// What the values of N rows want from memory, all asked for before the first is used (a store in between could not be passed by a load).
// E: type of the operands, O: of the result.  Columns c .. c+3 and c+APART .. c+APART+3 of rows r, r + step, ..; `left` columns are there from c on,
// all eight if WHOLE.  (APART 4: eight together, 16 bytes of bf16.  In fp32 the halves are as far apart as makes the lanes of a row lie together.)
template <class E, class O, int N, bool WHOLE, int APART = 4> struct Finisher {
    const Finish& f;
    int64_t set;
    int c, left;
    float bias[8];

    template <class X> __device__ __forceinline__ void load(const X* p, float (&v)[8]) const {
        if (APART == 4) { load_some<X, 8>(p, WHOLE ? 8 : left, v); return; }
        float lo[4], hi[4];
        load_some<X, 4>(p, WHOLE ? 4 : left, lo);
        load_some<X, 4>(p + APART, WHOLE ? 4 : left - APART, hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) { v[k] = lo[k]; v[4 + k] = hi[k]; }
    }
    template <class X> __device__ __forceinline__ void store(X* p, const float (&v)[8]) const {
        if (APART == 4) { store_some<X, 8>(p, WHOLE ? 8 : left, v); return; }
        const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
        store_some<X, 4>(p, WHOLE ? 4 : left, lo);
        store_some<X, 4>(p + APART, WHOLE ? 4 : left - APART, hi);
    }

    __device__ __forceinline__ Finisher(const Finish& f, int64_t set, int c, int left) : f(f), set(set), c(c), left(left) {
        if (f.bias) load(f.bias + set * f.bias_set + c, bias);
    }
    // value(u, v): the eight values of row r + u * step; rows from `end` on are left out
    template <class Value> __device__ __forceinline__ void operator()(int64_t r, int step, int64_t end, Value value) const {
        if (!WHOLE && left <= 0) return;
        float before[N][8], residual[N][8];
        if (f.before) {
#pragma unroll
            for (int u = 0; u < N; ++u) if (r + u * step < end) load((const E*)f.before + set * f.before_set + (r + u * step) * f.before_row + c, before[u]);
        }
        if (f.residual) {
#pragma unroll
            for (int u = 0; u < N; ++u) if (r + u * step < end) load((const E*)f.residual + set * f.residual_set + (r + u * step) * f.residual_row + c, residual[u]);
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (r + u * step >= end) break;
            float v[8];
            value(u, v);
            if (f.bias) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] += bias[k];
            }
            if (f.kept) store((E*)f.kept + set * f.kept_set + (r + u * step) * f.kept_row + c, v);
            if (f.silu) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= sigmoid_of(v[k] * SILU_SCALE);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __builtin_elementwise_maximum(v[k], f.floor);
            }
            if (f.before) {
                if (f.slope_silu) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = through_slope<true>(v[k], before[u][k] * SILU_SCALE, 0.f);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = through_slope<false>(v[k], before[u][k], 0.f);
                }
            }
            if (f.residual) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] += residual[u][k];
            }
            store((O*)f.out + set * f.out_set + (r + u * step) * f.out_row + c, v);
        }
    }
};
#endif

}  // namespace kavg
