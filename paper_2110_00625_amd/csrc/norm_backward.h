// Backward pass of the group norm on tiles in registers (norm_tile.h).  With da = drop(dy), dz = da act'(z), z = weight_c xh + bias_c:
//     dbias_c = sum dz,  dweight_c = sum dz xh  over a learner's images and positions,
//     dx = r (weight_c dz - A - xh B),  A = mean weight_c dz,  B = mean weight_c dz xh  over the group.
// Everything is linear in dz: drop's scale and r (xh = (x - m) r) are applied to sums and parameters, not to elements.
// Both pairs come from the same sums, of dz and dz xh per channel of an image: they are taken once, the group's are the sum over its
// channels times their weights, and the parameters' the sum over images, by a kernel of its own (norm_param_kernel), in a fixed order.
// x and dz stay in registers between the sums and dx, so that x and dy are read once.  An image that one workgroup cannot hold is read
// twice: sums of its chunks, their sum, results.
#pragma once
#include "norm_tile.h"

namespace kavg {

struct BackwardCall {
    NormCall n;
    Tile t;
    int64_t x_extent, dy_extent;
    float* parts;                  // [image][chunk] of (sum dz [channels], sum dz xh [channels])
    const float* group_sums;       // [image][group] of (A, B): results from finished sums
};

template <int V> __device__ __forceinline__ void slopes(int activation, const float (&z)[V], float (&d)[V]) {
    if (activation == KAVG_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] *= activate_slope<KAVG_ACT_SILU>(z[i]);
    } else if (activation == KAVG_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] *= activate_slope<KAVG_ACT_RELU>(z[i]);
    }
}

template <class E, int V, int NV, bool FLAT, bool WHOLE_PACK, int MODE>
__global__ void __launch_bounds__(1024) norm_backward_kernel(BackwardCall f) {
    constexpr int A = WHOLE_PACK ? 1 : V;
    extern __shared__ float lds[];
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t);
    const int D = c.channels / c.groups, threads = blockDim.x;
    typename Pack<E, V>::type xv[NV], gv[NV];
    {
        const Place<V, FLAT> from(c, t, l, c.xs), at(c, t, l, c.dys);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            xv[k] = tile_load<E, V, FLAT>(t, l, (const E*)c.x, from, f.x_extent, k);
            gv[k] = tile_load<E, V, FLAT>(t, l, (const E*)c.dy, at, f.dy_extent, k);
        }
    }
    float w[V], b[V], mean[A], rstd[A];              // (w: weight_c r)
    int group[A];                                    // in the tile
    // (a lane without work, whose group may not exist, looks at the first one)
    const int64_t first_group = l.on ? (int64_t)l.image * c.groups + l.block * t.groups : 0;
#pragma unroll
    for (int a = 0; a < A; ++a) {
        group[a] = l.on ? fastdiv(FLAT ? l.channel(c, a) : l.col * V + a, t.d_m, t.d_s) : 0;
        mean[a] = c.mean[first_group + group[a]];
        rstd[a] = c.rstd[first_group + group[a]];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int ch = l.channel(c, i);
        w[i] = (c.weight ? c.weight[l.set * c.weight_stride + ch] : 1.f) * rstd[WHOLE_PACK ? 0 : i];
        b[i] = c.bias ? c.bias[l.set * c.bias_stride + ch] : 0.f;
    }
    const uint64_t number = l.number(c, t), number_step = l.number_step(c, t);
    // of pack k: x - m, and dz without drop's scale
    const auto gradient = [&](int k, float (&d)[V], float (&g)[V]) {
        float z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            d[i] = to_float(xv[k][i]) - mean[WHOLE_PACK ? 0 : i];
            z[i] = d[i] * w[i] + b[i];
            g[i] = to_float(gv[k][i]);
        }
        if (c.drop.threshold) tile_mask<V, FLAT>(c.drop, l.run, number + k * number_step, g);
        slopes<V>(c.activation, z, g);
    };

    float dz[MODE == TILE_WHOLE ? NV : 1][V];
    float gA[A], gB[A];                              // r A, r B
    if (MODE != TILE_APPLY) {
        float s0[V], s1[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s0[i] = s1[i] = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float d[V], (&g)[V] = dz[MODE == TILE_WHOLE ? k : 0];
            gradient(k, d, g);
            const int n = l.valid(t, k);
            if (n == V) {
#pragma unroll
                for (int i = 0; i < V; ++i) { s0[i] += g[i]; s1[i] += g[i] * d[i]; }
            } else if (FLAT && n) {
#pragma unroll
                for (int i = 0; i < V; ++i) if (i < n) { s0[i] += g[i]; s1[i] += g[i] * d[i]; }
            }
            keep_packed(xv[k]);
        }
        // over the tile's places, per channel: `shares` lanes a channel, then those
        const int tc = FLAT ? c.channels : t.channels, sums = t.units * tc, places = FLAT ? t.cols * V / c.channels : t.lane_rows;
        float* p0 = lds;                             // [lane][V]: [unit][place][channel]
        float* p1 = p0 + threads * V;
        float* q0 = p1 + threads * V;                // [share][unit][channel]
        float* q1 = q0 + threads;
        float* c0 = q1 + threads;                    // [unit][channel]
        float* c1 = c0 + sums;
        float* g0 = c1 + sums;                       // [unit][group]
        float* g1 = g0 + t.units * t.groups;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p0[threadIdx.x * V + i] = l.on ? s0[i] * c.drop.scale : 0.f;
            p1[threadIdx.x * V + i] = l.on ? s1[i] * (c.drop.scale * rstd[WHOLE_PACK ? 0 : i]) : 0.f;
        }
        __syncthreads();
        const int shares = sums >= threads ? 1 : places < threads / sums ? places : threads / sums;
        for (int s = threadIdx.x; s < sums * shares; s += threads) {
            const int share = s / sums, ch = s - share * sums, unit = ch / tc, base = unit * t.cols * t.lane_rows * V + ch - unit * tc;
            float a0 = 0.f, a1 = 0.f;
            for (int r = share; r < places; r += shares) { a0 += p0[base + r * tc]; a1 += p1[base + r * tc]; }
            (shares > 1 ? q0 : c0)[s] = a0;
            (shares > 1 ? q1 : c1)[s] = a1;
        }
        __syncthreads();
        const int64_t image0 = (int64_t)l.image - l.unit, images = c.sets * c.images;
        for (int ch = threadIdx.x; ch < sums; ch += threads) {
            float a0 = c0[ch], a1 = c1[ch];
            if (shares > 1) {
                a0 = a1 = 0.f;
                for (int s = 0; s < shares; ++s) { a0 += q0[s * sums + ch]; a1 += q1[s * sums + ch]; }
                c0[ch] = a0;
                c1[ch] = a1;
            }
            const int unit = ch / tc, in = (int)l.block * t.channels + ch - unit * tc;
            if (f.parts && image0 + unit < images && in < c.channels) {
                float* to = f.parts + ((image0 + unit) * t.chunks + l.chunk) * 2 * c.channels + in;
                to[0] = a0;
                to[c.channels] = a1;
            }
        }
        if (MODE == TILE_SUMS) return;
        __syncthreads();
        const int groups = t.units * t.groups, team = team_of(threads, groups, D), lane = threadIdx.x % team;
        const float n = (float)c.positions * (float)D;
        for (int g = threadIdx.x / team; g < groups; g += threads / team) {
            const int unit = g / t.groups, in = (g - unit * t.groups) * D, ch0 = (int)l.block * t.channels + in;
            const int64_t image = image0 + unit;
            float a0 = 0.f, a1 = 0.f;
            if (image < images && ch0 < c.channels) {
                const float* weight = c.weight ? c.weight + image / c.images * c.weight_stride + ch0 : nullptr;
                for (int i = lane; i < D; i += team) {
                    const float wi = weight ? weight[i] : 1.f;
                    a0 += wi * c0[unit * tc + in + i];
                    a1 += wi * c1[unit * tc + in + i];
                }
            }
            a0 = team_sum(a0, team);
            a1 = team_sum(a1, team);
            if (lane == 0) { g0[g] = a0 / n; g1[g] = a1 / n; }
        }
        __syncthreads();
#pragma unroll
        for (int a = 0; a < A; ++a) {
            gA[a] = rstd[a] * g0[l.unit * t.groups + group[a]];
            gB[a] = rstd[a] * g1[l.unit * t.groups + group[a]];
        }
    } else {
#pragma unroll
        for (int a = 0; a < A; ++a) {
            gA[a] = rstd[a] * f.group_sums[2 * (first_group + group[a])];
            gB[a] = rstd[a] * f.group_sums[2 * (first_group + group[a]) + 1];
        }
    }
    const Place<V, FLAT> to(c, t, l, c.outs);
#pragma unroll
    for (int a = 0; a < A; ++a) gB[a] *= rstd[a];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float v[V], d[V];
        if (MODE == TILE_APPLY) gradient(k, d, v);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int a = WHOLE_PACK ? 0 : i;
            if (MODE == TILE_WHOLE) { v[i] = dz[k][i]; d[i] = to_float(xv[k][i]) - mean[a]; }
            v[i] = v[i] * (w[i] * c.drop.scale) - gA[a] - d[i] * gB[a];
        }
        tile_store<E, V, FLAT>(t, l, (E*)c.out, to, k, v);
    }
}

template <class E> hipError_t tiled_backward(const NormCall& c, const Tile& t, void* workspace, hipStream_t st);

}  // namespace kavg
