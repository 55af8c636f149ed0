// Forward pass of the group norm on tiles in registers (norm_tile.h):
//     m = mean x,  v = mean (x - m)^2,  r = (v + eps)^(-1/2),  y = drop(act(weight_c r (x - m) + bias_c)).
// A lane takes mean and squared distances from it of its own elements (per group, or per channel where a pack straddles groups), the
// lanes of a group are joined as means of parts: m = sum n_i m_i / n, n v = sum (q_i + n_i (m_i - m)^2), which loses nothing where the
// mean is far from zero.  Images cut into chunks leave (m, n v) of every chunk and are joined the same way by a kernel of their own.
#pragma once
#include "norm_tile.h"

namespace kavg {

struct ForwardCall {
    NormCall n;
    Tile t;
    int64_t x_extent;
    float* parts;          // [image][group][chunk] of (mean, squares), chunks only
    const float *mean, *rstd;      // results from finished sums
};

template <class E, int V, int NV, bool FLAT, bool WHOLE_PACK, int MODE>
__global__ void __launch_bounds__(1024) norm_forward_kernel(ForwardCall f) {
    constexpr int A = WHOLE_PACK ? 1 : V;            // sums of a lane
    extern __shared__ float lds[];
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t);
    const int D = c.channels / c.groups;
    const Place<V, FLAT> from(c, t, l, c.xs);
    typename Pack<E, V>::type xv[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) xv[k] = tile_load<E, V, FLAT>(t, l, (const E*)c.x, from, f.x_extent, k);

    float w[V], b[V];
    const auto parameters = [&] {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int ch = l.channel(c, i);
            w[i] = c.weight ? c.weight[l.set * c.weight_stride + ch] : 1.f;
            b[i] = c.bias ? c.bias[l.set * c.bias_stride + ch] : 0.f;
        }
    };
    int group[A];                                    // in the tile
#pragma unroll
    for (int a = 0; a < A; ++a) group[a] = fastdiv(FLAT ? l.channel(c, a) : l.col * V + a, t.d_m, t.d_s);
    float mean[A], rstd[A];

    if (MODE != TILE_APPLY) {
        const int threads = blockDim.x;
        float* part_sum = lds;                       // [lane][A]
        float* part_sq = lds + threads * A;
        float* stat = part_sq + threads * A;         // [unit][group of the tile] mean, then rstd
        // of the chunk: whole rounds of the lanes, and rows (flat: elements) of the last one
        const int64_t all = FLAT ? l.run : t.rows, step = FLAT ? (int64_t)t.cols * V : t.lane_rows;
        const int64_t before = (int64_t)l.chunk * NV * step, here = all - before < NV * step ? all - before : NV * step;
        const int rounds = (int)(here / step), rest = (int)(here - rounds * step);
        float sum[A], sq[A];
#pragma unroll
        for (int a = 0; a < A; ++a) sum[a] = sq[a] = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int n = l.valid(t, k);
            if (WHOLE_PACK) { if (n) sum[0] = pack_sum<V>(xv[k], sum[0]); }
            else if (n == V) {
#pragma unroll
                for (int i = 0; i < V; ++i) sum[WHOLE_PACK ? 0 : i] += to_float(xv[k][i]);
            } else if (FLAT && n) {
#pragma unroll
                for (int i = 0; i < V; ++i) sum[WHOLE_PACK ? 0 : i] += i < n ? to_float(xv[k][i]) : 0.f;
            }
            keep_packed(xv[k]);
        }
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const int n = l.on ? (rounds + ((FLAT ? (int)l.col * V + a : (int)l.row) < rest)) * (WHOLE_PACK ? V : 1) : 0;
            mean[a] = n ? sum[a] / (float)n : 0.f;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int n = l.valid(t, k);
            if (n == V) {
#pragma unroll
                for (int i = 0; i < V; ++i) { const float d = to_float(xv[k][i]) - mean[WHOLE_PACK ? 0 : i]; sq[WHOLE_PACK ? 0 : i] += d * d; }
            } else if (FLAT && n) {
#pragma unroll
                for (int i = 0; i < V; ++i) if (i < n) { const float d = to_float(xv[k][i]) - mean[WHOLE_PACK ? 0 : i]; sq[WHOLE_PACK ? 0 : i] += d * d; }
            }
            keep_packed(xv[k]);
        }
#pragma unroll
        for (int a = 0; a < A; ++a) { part_sum[threadIdx.x * A + a] = sum[a]; part_sq[threadIdx.x * A + a] = sq[a]; }
        if (MODE != TILE_SUMS) parameters();         // (on their way while the groups are joined)
        __syncthreads();
        // a team of lanes per group: parts (place, channel or pack) of the group, row by row
        const int per = WHOLE_PACK ? D / V : D, slots = (FLAT ? c.channels : t.channels) / (WHOLE_PACK ? V : 1);
        const int places = FLAT ? t.cols * V / c.channels : t.lane_rows, terms = places * per, sums = t.units * t.groups;
        const int team = team_of(threads, sums, terms), lane = threadIdx.x % team;
        const float n = (float)(FLAT ? here / c.channels : here) * (float)D;
        for (int g = threadIdx.x / team; g < sums; g += threads / team) {
            const int unit = g / t.groups, in = g - unit * t.groups, base = unit * t.cols * t.lane_rows * A + in * per;
            float s = 0.f;
            for (int j = lane, r = lane / per, i = lane - r * per; j < terms; j += team) {
                s += part_sum[base + r * slots + i];
                i += team;
                while (i >= per) { i -= per; ++r; }
            }
            const float m = team_sum(s, team) / n;
            float q = 0.f;
            for (int j = lane, r = lane / per, i = lane - r * per; j < terms; j += team) {
                const int place = FLAT ? r * slots + in * per + i : r;
                const float cnt = (float)((rounds + (place < rest)) * (WHOLE_PACK ? V : 1));
                const float d = cnt > 0.f ? part_sum[base + r * slots + i] / cnt - m : 0.f;
                q += part_sq[base + r * slots + i] + cnt * d * d;
                i += team;
                while (i >= per) { i -= per; ++r; }
            }
            q = team_sum(q, team);
            if (lane == 0) {
                const int64_t image = (int64_t)l.image - l.unit + unit;
                const int group_ = (int)l.block * t.groups + in;
                const bool there = image < c.sets * c.images && group_ < c.groups;
                const int64_t at = image * c.groups + group_;
                if (MODE == TILE_SUMS) {
                    if (there) { f.parts[(at * t.chunks + l.chunk) * 2] = m; f.parts[(at * t.chunks + l.chunk) * 2 + 1] = q; }
                } else {
                    const float rs = 1.f / sqrtf(q / n + c.eps);
                    stat[g] = m;
                    stat[sums + g] = rs;
                    if (c.mean && there) { c.mean[at] = m; c.rstd[at] = rs; }
                }
            }
        }
        if (MODE == TILE_SUMS) return;
        __syncthreads();
#pragma unroll
        for (int a = 0; a < A; ++a) { mean[a] = stat[l.unit * t.groups + group[a]]; rstd[a] = stat[sums + l.unit * t.groups + group[a]]; }
    } else {
        parameters();
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const int64_t at = l.on ? (int64_t)l.image * c.groups + l.block * t.groups + group[a] : 0;
            mean[a] = f.mean[at];
            rstd[a] = f.rstd[at];
        }
    }
    const Place<V, FLAT> to(c, t, l, c.outs);
    const uint64_t number = l.number(c, t), number_step = l.number_step(c, t);
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] *= rstd[WHOLE_PACK ? 0 : i];
    // drop's scale commutes with ReLU
    if (c.activation != KAVG_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < V; ++i) { w[i] *= c.drop.scale; b[i] *= c.drop.scale; }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (to_float(xv[k][i]) - mean[WHOLE_PACK ? 0 : i]) * w[i] + b[i];
        if (c.activation == KAVG_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activate<KAVG_ACT_SILU>(v[i]) * c.drop.scale;
        } else if (c.activation == KAVG_ACT_RELU) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activate<KAVG_ACT_RELU>(v[i]);
        }
        if (c.drop.threshold) tile_mask<V, FLAT>(c.drop, l.run, number + k * number_step, v);
        tile_store<E, V, FLAT>(t, l, (E*)c.out, to, k, v);
    }
}

// mean and 1/sqrt(v + eps) of a group from its chunks: a wavefront per group
template <int T>
__global__ void __launch_bounds__(T) norm_join_kernel(const float* parts, int chunks, int64_t groups, float whole, float last, float eps, float* mean, float* rstd,
                                                      float* mean2, float* rstd2) {
    const int64_t g = (int64_t)blockIdx.x * (T / 64) + threadIdx.x / 64;
    const int lane = threadIdx.x % 64;
    if (g >= groups) return;
    const float2* p = (const float2*)parts + g * chunks;
    const float n = whole * (float)(chunks - 1) + last;
    float s = 0.f;
    for (int i = lane; i < chunks; i += 64) s += p[i].x * (i < chunks - 1 ? whole : last);
    const float m = team_sum(s, 64) / n;
    float q = 0.f;
    for (int i = lane; i < chunks; i += 64) { const float d = p[i].x - m; q += p[i].y + (i < chunks - 1 ? whole : last) * d * d; }
    q = team_sum(q, 64);
    if (lane == 0) {
        const float r = 1.f / sqrtf(q / n + eps);
        mean[g] = m;
        rstd[g] = r;
        if (mean2) { mean2[g] = m; rstd2[g] = r; }
    }
}

template <class E> hipError_t tiled_forward(const NormCall& c, const Tile& t, void* workspace, hipStream_t st);

}  // namespace kavg
