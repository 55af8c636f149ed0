// Forward pass of the group norm on tiles in registers (norm_tile.h):
//     m = mean x,  v = mean (x - m)^2,  r = (v + eps)^(-1/2),  y = drop(act(weight_c r (x - m) + bias_c)).
// A lane takes mean and squared distances from it of its own elements (per group, or per channel where a pack straddles groups), the
// lanes of a group are joined as means of parts: m = sum n_i m_i / n, n v = sum (q_i + n_i (m_i - m)^2), which loses nothing where the
// mean is far from zero.  The chunks of an image that is read twice, and the turns of a chunk, are joined the same way.
#pragma once
#include "norm_tile.h"

namespace kavg {

struct ForwardCall {
    NormCall n;
    Tile t;
    int64_t x_extent;
    float* parts;                  // [image][group][chunk] of (mean, squares)
    // results from finished sums: mean and rstd, or, where they are null, the parts of `chunks` chunks, all but the last of `whole` values
    const float *mean, *rstd;
    int chunks;
    float whole, last;
};

// mean and sum of squared distances of a group's values from its parts: a team of lanes, part j with n(j) values, mean m(j), squares q(j)
template <class N, class M, class Q>
__device__ __forceinline__ void join_parts(int terms, int lane, int team, float n, N count, M mean_of, Q squares_of, float* mean, float* squares) {
    float s = 0.f;
    for (int j = lane; j < terms; j += team) s += count(j) * mean_of(j);
    const float m = team_sum(s, team) / n;
    float q = 0.f;
    for (int j = lane; j < terms; j += team) { const float d = mean_of(j) - m; q += squares_of(j) + count(j) * d * d; }
    *mean = m;
    *squares = team_sum(q, team);
}

// mean[a], sq[a]: of a lane's NV packs (flat: of each of their elements; GRAN elements of a pack otherwise) their mean and squared distances
// from it.  All NV packs are the image's.
template <class E, int V, int NV, int GRAN>
__device__ __forceinline__ void whole_moments(const typename Pack<E, V>::type (&xv)[NV], float (&mean)[V / GRAN], float (&sq)[V / GRAN]) {
    constexpr int A = V / GRAN;
    float sum[A];
#pragma unroll
    for (int a = 0; a < A; ++a) sum[a] = sq[a] = 0.f;
    const auto add_distances = [&](float (&to)[A]) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            auto v = xv[k];
            keep_packed(v);
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = to_float(v[i]) - mean[i / GRAN]; to[i / GRAN] += d * d; }
        }
    };
    if constexpr (sizeof(E) == 2 && GRAN > 1) {
        // bf16: sums of values and of squares by dot products (half an instruction per element each; a mean and distances from it are four).
        // n v = sum x^2 - n m^2 cancels where the mean is large against the spread: a sum that loses more than two bits is taken of the
        // distances after all, each for itself, so that no group's result depends on another one's values.
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int a = 0; a < A; ++a) { sum[a] = pack_sum<GRAN>(xv[k], a * GRAN, sum[a]); sq[a] = pack_squares<GRAN>(xv[k], a * GRAN, sq[a]); }
        }
        bool lost[A], any = false;
#pragma unroll
        for (int a = 0; a < A; ++a) {
            mean[a] = sum[a] * (1.f / (NV * GRAN));
            const float all = sq[a];
            sq[a] = all - sum[a] * mean[a];
            lost[a] = !(__builtin_fmaf(-0.25f, all, sq[a]) >= 0.f);         // (squares whose sum overflows: NaN, and lost)
            any |= lost[a];
        }
        if (!__any(any)) return;
        float far[A];
#pragma unroll
        for (int a = 0; a < A; ++a) far[a] = 0.f;
        add_distances(far);
#pragma unroll
        for (int a = 0; a < A; ++a) sq[a] = lost[a] ? far[a] : sq[a];
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int a = 0; a < A; ++a) sum[a] = pack_sum<GRAN>(xv[k], a * GRAN, sum[a]);
        }
#pragma unroll
        for (int a = 0; a < A; ++a) mean[a] = sum[a] * (1.f / (NV * GRAN));
        add_distances(sq);
    }
}

// The same of packs from the `first`-th on of which not all are the image's, and how many are (flat: of each element): `whole` of them, and one
// more in some lanes (flat: or a part of one).
template <class E, int V, int NV, bool FLAT, int GRAN>
__device__ __forceinline__ void lane_moments(const typename Pack<E, V>::type (&xv)[NV], const Tile& t, const Lane<V, FLAT>& l, int first, float (&mean)[V / GRAN],
                                             float (&sq)[V / GRAN], float (&count)[FLAT ? V : 1]) {
    constexpr int A = V / GRAN;
    int whole = 0, more = 0;                         // more: elements of the pack behind the whole ones
    float sum[A];
#pragma unroll
    for (int a = 0; a < A; ++a) sum[a] = sq[a] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (l.whole(t, first + k)) {
            ++whole;
#pragma unroll
            for (int a = 0; a < A; ++a) sum[a] = pack_sum<GRAN>(xv[k], a * GRAN, sum[a]);
        } else {
            const int n = l.valid(t, first + k);
            more |= n;                               // (no other pack has any)
            if (FLAT) {
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i / GRAN] += i < n ? to_float(xv[k][i]) : 0.f;
            } else if (n) {
#pragma unroll
                for (int a = 0; a < A; ++a) sum[a] = pack_sum<GRAN>(xv[k], a * GRAN, sum[a]);
            }
        }
    }
    const float each = whole ? 1.f / (float)(whole * GRAN) : 0.f, each_more = 1.f / (float)((whole + 1) * GRAN);
#pragma unroll
    for (int a = 0; a < A; ++a) mean[a] = sum[a] * ((FLAT ? a : 0) < more ? each_more : each);
#pragma unroll
    for (int a = 0; a < (FLAT ? V : 1); ++a) count[a] = (float)(whole + (a < more));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        auto v = xv[k];
        keep_packed(v);
        if (l.whole(t, first + k)) {
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = to_float(v[i]) - mean[i / GRAN]; sq[i / GRAN] += d * d; }
        } else {
            const int n = l.valid(t, first + k);
            if (n) {
#pragma unroll
                for (int i = 0; i < V; ++i) { const float d = to_float(v[i]) - mean[i / GRAN]; sq[i / GRAN] += !FLAT || i < n ? d * d : 0.f; }
            }
        }
    }
}

// The lanes' moments joined per group of the tile: done(unit, group in the tile, mean, squares) in one lane of each.  lds: 2 * lanes * A floats.
template <int V, bool FLAT, int GRAN, class Done>
__device__ __forceinline__ void join_lanes(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l, const Chunk<V, FLAT>& chunk, float* lds,
                                           const float (&mean)[V / GRAN], const float (&sq)[V / GRAN], Done done) {
    constexpr int A = V / GRAN;
    const int threads = blockDim.x, D = c.channels / c.groups;
    float* part_mean = lds;                          // [lane][A]: [unit][place][channel or pack]
    float* part_sq = lds + threads * A;
#pragma unroll
    for (int a = 0; a < A; ++a) { part_mean[threadIdx.x * A + a] = mean[a]; part_sq[threadIdx.x * A + a] = sq[a]; }
    __syncthreads();
    const int per = D / GRAN, slots = (FLAT ? c.channels : t.channels) / GRAN;
    const int places = FLAT ? t.cols * V / c.channels : t.lane_rows, terms = places * per, groups = t.units * t.groups;
    const int team = team_of(threads, groups, terms), lane = threadIdx.x % team;
    for (int g = threadIdx.x / team; g < groups; g += threads / team) {
        const int unit = g / t.groups, in = g - unit * t.groups, base = unit * t.cols * t.lane_rows * A + in * per;
        // part j of the group: place j / per
        const auto place = [&](int j) { return (int)divide(j, t.by_per); };
        const auto slot = [&](int j) { const int r = place(j); return r * slots + j - r * per; };
        float m, q;
        join_parts(terms, lane, team, chunk.positions * (float)D,
                   [&](int j) { return (float)(chunk.rounds_of(FLAT ? slot(j) + in * per : place(j)) * GRAN); },
                   [&](int j) { return part_mean[base + slot(j)]; }, [&](int j) { return part_sq[base + slot(j)]; }, &m, &q);
        if (lane == 0) done(unit, in, m, q);
    }
}

// weight times r; SiLU's factor into both, or drop's scale, which commutes with ReLU
template <int V, int GRAN, bool SILU, bool DROP>
__device__ __forceinline__ void scale_parameters(const NormCall& c, const float (&rstd)[V / GRAN], float (&w)[V], float (&b)[V]) {
    const float scale = SILU ? SILU_SCALE : c.drop.scale;
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] *= rstd[i / GRAN];
    if (DROP || SILU) {
#pragma unroll
        for (int i = 0; i < V; ++i) { w[i] *= scale; b[i] *= scale; }
    }
}

// y of pack k
template <class E, int V, bool FLAT, int GRAN, bool SILU, bool DROP>
__device__ __forceinline__ void write_result(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l, const Place<V, FLAT>& to, int k, const TileMask<V, FLAT>& mask,
                                             const typename Pack<E, V>::type& x, const float (&mean)[V / GRAN], const float (&w)[V], const float (&b)[V]) {
    const float after = SILU_BACK * (DROP ? c.drop.scale : 1.f);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i] = activate<SILU>((to_float(x[i]) - mean[i / GRAN]) * w[i] + b[i], c.floor);
        if (SILU) v[i] *= after;
    }
    typename Pack<E, V>::type o = packed<E, V>(v);
    if (DROP) mask.template drop<E>(c.drop, k, o);
    tile_store<E, V, FLAT>(t, l, (E*)c.out, to, k, o);
}

// Images that a workgroup holds: read once, statistics, result, written once.  Up to sixteen packs per lane, so that two workgroups of 512 lanes
// with 64 KB of x each share a compute unit and one loads while the other computes or writes.  Bound by memory where there is much: 1024 images of
// 32x32x128 in bf16 with ReLU and dropout 111 us, 4.8 TB/s (a copy of that size 5.1), 15 vector instructions per element, half of them the
// draws'.  A thousand vectors of 1024 in fp32: 7.0 us, a launch and its latencies.
template <class E, int V, int NV, bool FLAT, int GRAN, bool SILU, bool DROP>
__global__ void __launch_bounds__(1024) norm_forward_kernel(ForwardCall f) {
    constexpr int A = V / GRAN;
    extern __shared__ float lds[];
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t, tile_of_workgroup(gridDim.x));
    typename Pack<E, V>::type xv[NV];
    {
        const Place<V, FLAT> from(c, t, l, c.xs);
        load_packs<NV>(t, l, 0, [&](int k, auto whole) { xv[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.x, from, f.x_extent, k); });
    }
    const Chunk<V, FLAT> chunk(c, t, l);
    float mean[A], rstd[A], w[V], b[V];
    int group[A];
    constexpr bool ASK = GRAN > 1 || NV <= FLAT_PACKS;      // (both ways of sixteen packs with sums per channel do not fit the registers)
    if (ASK && l.whole(t, NV - 1)) whole_moments<E, V, NV, GRAN>(xv, mean, rstd);
    else {
        float count[FLAT ? V : 1];
        lane_moments<E, V, NV, FLAT, GRAN>(xv, t, l, 0, mean, rstd, count);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) keep_packed(xv[k]);
    lane_parameters(c, t, l, w, b, group);                     // (on their way while the groups are joined)
    float* stat = lds + 2 * blockDim.x * A;          // [unit][group of the tile] mean, then rstd
    const int groups = t.units * t.groups, D = c.channels / c.groups;
    join_lanes<V, FLAT, GRAN>(c, t, l, chunk, lds, mean, rstd, [&](int unit, int in, float m, float q) {
        const float r = 1.f / sqrtf(q / (chunk.positions * (float)D) + c.eps);
        stat[unit * t.groups + in] = m;
        stat[groups + unit * t.groups + in] = r;
        const uint32_t image = l.first_image + unit;
        const int g = (int)l.block * t.groups + in;
        if (c.mean && image < (uint32_t)(c.sets * c.images) && g < c.groups) {
            c.mean[(int64_t)image * c.groups + g] = m;
            c.rstd[(int64_t)image * c.groups + g] = r;
        }
    });
    __syncthreads();
#pragma unroll
    for (int a = 0; a < A; ++a) { mean[a] = stat[l.unit * t.groups + group[a]]; rstd[a] = stat[groups + l.unit * t.groups + group[a]]; }
    scale_parameters<V, GRAN, SILU, DROP>(c, rstd, w, b);
    const Place<V, FLAT> to(c, t, l, c.outs);
    const TileMask<V, FLAT> mask(c, t, l);
#pragma unroll
    for (int k = 0; k < NV; ++k) write_result<E, V, FLAT, GRAN, SILU, DROP>(c, t, l, to, k, mask, xv[k], mean, w, b);
}

// Moments of a chunk, in turns of SUM_PACKS packs per lane, the next turn's on their way; a lane joins its turns as means of parts.  Bound by
// latency: of 33 MB (two images of 256x256x128 in bf16) 11.0 us, 3.0 TB/s, a load, two turns and the join of the lanes.
template <class E, int V, bool FLAT, int GRAN>
__global__ void __launch_bounds__(512) norm_moments_kernel(ForwardCall f) {
    constexpr int A = V / GRAN, NV = SUM_PACKS;
    extern __shared__ float lds[];
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t, tile_of_workgroup(gridDim.x));
    const Place<V, FLAT> from(c, t, l, c.xs);
    typename Pack<E, V>::type next[NV];
    const auto packs_from = [&](int first) {
        load_packs<NV>(t, l, first, [&](int k, auto whole) { next[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.x, from, f.x_extent, first + k); });
    };
    packs_from(0);
    float mean[A], sq[A];
#pragma unroll
    for (int a = 0; a < A; ++a) mean[a] = sq[a] = 0.f;
    for (int turn = 0; turn < t.nv; turn += NV) {
        typename Pack<E, V>::type xv[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) xv[k] = next[k];
        if (turn + NV < t.nv) packs_from(turn + NV);
        float m[A], q[A];
        if (l.whole(t, turn + NV - 1)) {
            whole_moments<E, V, NV, GRAN>(xv, m, q);
            const float old = (float)(turn * GRAN), share = (NV * GRAN) / (old + NV * GRAN), both = old * share;
#pragma unroll
            for (int a = 0; a < A; ++a) {
                const float d = m[a] - mean[a];
                mean[a] += d * share;
                sq[a] += q[a] + d * d * both;
            }
            continue;
        }
        // (the image ends in this turn or did before: the turns in front of its end were whole)
        float count[FLAT ? V : 1];
        lane_moments<E, V, NV, FLAT, GRAN>(xv, t, l, turn, m, q, count);
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const float n = count[FLAT ? a : 0] * GRAN, old = (float)(turn * GRAN);
            const float share = n > 0.f ? n / (n + old) : 0.f, d = m[a] - mean[a];
            mean[a] += d * share;
            sq[a] += q[a] + d * d * (old * share);
        }
    }
    const Chunk<V, FLAT> chunk(c, t, l);
    join_lanes<V, FLAT, GRAN>(c, t, l, chunk, lds, mean, sq, [&](int unit, int in, float m, float q) {
        const int g = (int)l.block * t.groups + in;
        if (g >= c.groups) return;
        float* to = f.parts + (((int64_t)l.image * c.groups + g) * t.chunks + l.chunk) * 2;
        to[0] = m;
        to[1] = q;
    });
}

// Mean and 1/sqrt(v + eps) of a group from its chunks: a wavefront per group.  Only where the chunks are more than the workgroups of the results
// should join, each for itself; a launch and its latency, 4 us.
template <int T>
__global__ void __launch_bounds__(T) norm_join_kernel(ForwardCall f, int64_t groups, float* mean, float* rstd) {
    const int64_t g = (int64_t)blockIdx.x * (T / 64) + threadIdx.x / 64;
    if (g >= groups) return;
    float m, q;
    const float2* p = (const float2*)f.parts + g * f.chunks;
    const float all = f.whole * (float)(f.chunks - 1) + f.last;
    join_parts(f.chunks, threadIdx.x % 64, 64, all, [&](int j) { return j < f.chunks - 1 ? f.whole : f.last; },
               [&](int j) { return p[j].x; }, [&](int j) { return p[j].y; }, &m, &q);
    if (threadIdx.x % 64) return;
    const float r = 1.f / sqrtf(q / all + f.n.eps);
    mean[g] = m;
    rstd[g] = r;
    if (f.n.mean) { f.n.mean[g] = m; f.n.rstd[g] = r; }
}

// Results of an image read again, by the workgroups that read the same tiles for the sums, on the same XCD and the last first: those are
// what its cache still holds.  Those 33 MB read and written in 14.8 us, 4.5 TB/s.  (Images kept on chip from the sums to the results would want
// workgroups that wait for each other, which a caller's other work on the device could keep from running.)
template <class E, int V, bool FLAT, int GRAN, bool SILU, bool DROP>
__global__ void __launch_bounds__(512) norm_apply_kernel(ForwardCall f) {
    constexpr int A = V / GRAN, NV = APPLY_PACKS;
    extern __shared__ float lds[];
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t, tile_of_workgroup(gridDim.x, true));
    const Place<V, FLAT> from(c, t, l, c.xs), to(c, t, l, c.outs);
    // (loads return in order: what the first pack needs is asked for before the packs)
    float mean[A], rstd[A], w[V], b[V];
    int group[A];
    lane_parameters(c, t, l, w, b, group);
    typename Pack<E, V>::type next[NV];
    const auto packs_from = [&](int first) {
        load_packs<NV>(t, l, first, [&](int k, auto whole) { next[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.x, from, f.x_extent, first + k); });
    };
    const int64_t first = l.groups_at(c, t);
    if (f.mean) {
#pragma unroll
        for (int a = 0; a < A; ++a) { mean[a] = l.on ? f.mean[first + group[a]] : 0.f; rstd[a] = l.on ? f.rstd[first + group[a]] : 0.f; }
        packs_from(t.nv - NV);
    } else {
        // every workgroup joins the chunks of its groups, JOINED_PARTS of them per lane at most
        const int team = team_of(blockDim.x, t.groups, f.chunks), lane = threadIdx.x % team;
        const float all = f.whole * (float)(f.chunks - 1) + f.last;
        bool asked = false;
        for (int g = threadIdx.x / team; g < t.groups || !asked; g += blockDim.x / team) {
            const bool there = g < t.groups && (int)l.block * t.groups + g < c.groups;
            const float2* parts = (const float2*)f.parts + (there ? (first + g) * f.chunks : 0);
            float2 p[JOINED_PARTS];
            float n[JOINED_PARTS];
#pragma unroll
            for (int j = 0; j < JOINED_PARTS; ++j) {
                const int i = lane + j * team;
                p[j] = parts[i < f.chunks ? i : 0];
                n[j] = i < f.chunks - 1 ? f.whole : i < f.chunks ? f.last : 0.f;
            }
            if (!asked) packs_from(t.nv - NV);               // (behind the parts, which come first)
            asked = true;
            float s = 0.f, q = 0.f;
#pragma unroll
            for (int j = 0; j < JOINED_PARTS; ++j) if (n[j] > 0.f) s += n[j] * p[j].x;
            const float m = team_sum(s, team) / all;
#pragma unroll
            for (int j = 0; j < JOINED_PARTS; ++j) if (n[j] > 0.f) q += p[j].y + n[j] * (p[j].x - m) * (p[j].x - m);
            q = team_sum(q, team);
            if (lane || !there) continue;
            const float r = 1.f / sqrtf(q / all + c.eps);
            lds[g] = m;
            lds[t.groups + g] = r;
            if (c.mean && l.chunk == 0) { c.mean[first + g] = m; c.rstd[first + g] = r; }
        }
        __syncthreads();
#pragma unroll
        for (int a = 0; a < A; ++a) { mean[a] = lds[group[a]]; rstd[a] = lds[t.groups + group[a]]; }
    }
    scale_parameters<V, GRAN, SILU, DROP>(c, rstd, w, b);
    const TileMask<V, FLAT> mask(c, t, l);
    for (int turn = t.nv - NV; turn >= 0; turn -= NV) {
        typename Pack<E, V>::type xv[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) xv[k] = next[k];
        if (turn) packs_from(turn - NV);
#pragma unroll
        for (int k = 0; k < NV; ++k) write_result<E, V, FLAT, GRAN, SILU, DROP>(c, t, l, to, turn + k, mask, xv[k], mean, w, b);
    }
}

// ---- launches ----

template <class Kernel>
hipError_t start_forward(Kernel kernel, const ForwardCall& f, size_t lds, hipStream_t st) {
    const Tile& t = f.t;
    const int64_t images = f.n.sets * f.n.images, tiles = (images + t.units - 1) / t.units * t.blocks * t.chunks;
    if (lds > LDS_PLAIN) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)tiles), dim3(t.threads), lds, st>>>(f);
    return hipGetLastError();
}

template <class E, int V, bool FLAT, int GRAN>
hipError_t forward_twice(ForwardCall& f, const NormTiles& t, float* workspace, hipStream_t st) {
    const NormCall& c = f.n;
    const int64_t groups = c.sets * c.images * c.groups, whole = chunk_positions(c, t.sums);
    const float D = (float)(c.channels / c.groups);
    f.parts = workspace;
    f.chunks = t.sums.chunks;
    f.whole = (float)whole * D;
    f.last = (float)(c.positions - whole * (f.chunks - 1)) * D;
    f.t = t.sums;
    hipError_t e = start_forward(norm_moments_kernel<E, V, FLAT, GRAN>, f, f.t.lds, st);
    if (e != hipSuccess) return e;
    // The workgroups that write the results join the chunks of their groups themselves, where that is little beside their tile.
    if (f.chunks > JOINED_PARTS * team_of(t.apply.threads, t.apply.groups, f.chunks)) {
        float* mean = workspace + 2 * groups * f.chunks;
        f.mean = mean;
        f.rstd = mean + groups;
        norm_join_kernel<256><<<dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, st>>>(f, groups, mean, mean + groups);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    f.t = t.apply;
    return with_options(c, [&](auto silu, auto drop) {
        return start_forward(norm_apply_kernel<E, V, FLAT, GRAN, silu.value, drop.value>, f, 2 * f.t.groups * sizeof(float), st);
    });
}

template <class E, int V, int NV, bool FLAT, int GRAN>
hipError_t forward_whole(const ForwardCall& f, hipStream_t st) {
    return with_options(f.n, [&](auto silu, auto drop) {
        return start_forward(norm_forward_kernel<E, V, NV, FLAT, GRAN, silu.value, drop.value>, f, f.t.lds, st);
    });
}

template <class E> hipError_t tiled_forward(const NormCall& c, const NormTiles& tiles, void* workspace, hipStream_t st) {
    ForwardCall f = {};
    f.n = c;
    f.x_extent = extent_of(c, c.xs);
    const bool whole = tiles.whole.nv != 0;
    f.t = whole ? tiles.whole : tiles.sums;
    return with_layout<E>(f.t, [&](auto vec, auto flat, auto gran) {
        constexpr int V = vec.value;
        constexpr int G = gran.value;
        constexpr bool FLAT = flat.value;
        if (!whole) return forward_twice<E, V, FLAT, G>(f, tiles, (float*)workspace, st);
        switch (f.t.nv) {
            case 1: return forward_whole<E, V, 1, FLAT, G>(f, st);
            case 2: return forward_whole<E, V, 2, FLAT, G>(f, st);
            case 4: return forward_whole<E, V, 4, FLAT, G>(f, st);
            case 8: return forward_whole<E, V, 8, FLAT, G>(f, st);
            default: return forward_whole<E, V, FLAT ? FLAT_PACKS : FORWARD_PACKS, FLAT, G>(f, st);
        }
    });
}

}  // namespace kavg
