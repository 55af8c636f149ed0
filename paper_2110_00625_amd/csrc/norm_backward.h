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
    const float* group_sums;       // [image][group] of (A, B): results from finished sums, or null: from the parts of `chunks` chunks
    int chunks;
    uint32_t tiles;                // workgroups that write results; those behind them add up the parameters' gradients
    int param_wide, param_blocks;
};

// What a lane keeps of its channels: m, r, weight_c (then times r, and with bias_c SiLU's factor), bias_c.
template <int V, bool FLAT, int GRAN> struct Channels {
    static constexpr int A = V / GRAN;
    float w[V], b[V], mean[A], rstd[A];
    int group[A];                                    // in the tile
    int64_t first_group;                             // of the tile
    TileMask<V, FLAT> mask;

    __device__ __forceinline__ Channels(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l) : mask(c, t, l) {
        first_group = l.groups_at(c, t);
        lane_parameters(c, t, l, w, b, group);
#pragma unroll
        for (int a = 0; a < A; ++a) { mean[a] = c.mean[first_group + group[a]]; rstd[a] = c.rstd[first_group + group[a]]; }
    }
    // the tile's weights into LDS, by the lanes of the first place
    __device__ __forceinline__ void share(const Tile& t, const Lane<V, FLAT>& l, float* lds) const {
        if (l.on && l.row == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int ch = (int)l.col * V + i;
                if (!FLAT || ch < t.channels) lds[l.unit * t.channels + ch] = w[i];
            }
        }
    }
    template <bool SILU> __device__ __forceinline__ void scale() {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[i] *= rstd[i / GRAN];
            if (SILU) { w[i] *= SILU_SCALE; b[i] *= SILU_SCALE; }
        }
    }
    // what dx takes of its group: r A and r^2 B
    __device__ __forceinline__ void group_part(int a, float sum, float sum_xh, float (&rA)[A], float (&rrB)[A]) const {
        rrB[a] = rstd[a] * rstd[a] * sum_xh;
        rA[a] = rstd[a] * sum;
    }
    // of a pack: x - m
    template <class P> __device__ __forceinline__ void distances(const P& x, float (&d)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = to_float(x[i]) - mean[i / GRAN];
    }
    // of pack k: x - m, and dz without drop's scale
    template <class E, bool SILU, bool DROP>
    __device__ __forceinline__ void gradient(const NormCall& c, int k, const typename Pack<E, V>::type& x, typename Pack<E, V>::type dy, float (&d)[V], float (&g)[V]) const {
        if (DROP) mask.template drop<E>(c.drop, k, dy);
        float z[V];
        distances(x, d);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            z[i] = d[i] * w[i] + b[i];
            g[i] = to_float(dy[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = through_slope<SILU>(g[i], z[i], c.floor);
    }
};

// s0 += g, s1 += g d of a pack, n of its elements valid
template <int V, bool FLAT>
__device__ __forceinline__ void add_pack(int n, const float (&d)[V], const float (&g)[V], float (&s0)[V], float (&s1)[V]) {
    if (n == V) {
#pragma unroll
        for (int i = 0; i < V; ++i) { s0[i] += g[i]; s1[i] += g[i] * d[i]; }
    } else if (FLAT && n) {
#pragma unroll
        for (int i = 0; i < V; ++i) if (i < n) { s0[i] += g[i]; s1[i] += g[i] * d[i]; }
    }
}

// `shares` lanes for each of `sums` sums
KAVG_FD int shares_of(int threads, int sums, int terms) { return sums >= threads ? 1 : terms < threads / sums ? terms : threads / sums; }

// LDS of the sums
struct SumSpace {
    float *p0, *p1;          // [lane][V]: [unit][place][channel]
    float *q0, *q1;          // [share][unit][channel]
    float *c0, *c1;          // [unit][channel]: sums of dz, dz xh
    float* g0;               // [unit][group]: A, then B
    float* w;                // [unit][channel]: weights
    __device__ __forceinline__ SumSpace(float* lds, int packs, int sums, int groups, int threads) {
        p0 = lds;
        p1 = p0 + packs;
        q0 = p1 + packs;
        q1 = q0 + threads;
        c0 = q1 + threads;
        c1 = c0 + sums;
        g0 = c1 + sums;
        w = g0 + 2 * groups;
    }
};

// sums per channel from `terms` terms each, term(sum, j, &a0, &a1) adding the j-th: into c0, c1 and to done(sum, a0, a1)
template <class Term, class Done>
__device__ __forceinline__ void add_up(const SumSpace& s, int sums, int terms, Term term, Done done) {
    const int threads = blockDim.x, shares = shares_of(threads, sums, terms);
    if (shares > 1) {
        for (int i = threadIdx.x; i < sums * shares; i += threads) {
            const int share = (int)((uint32_t)i / (uint32_t)sums), sum = i - share * sums;
            float a0 = 0.f, a1 = 0.f;
#pragma unroll 4
            for (int j = share; j < terms; j += shares) term(sum, j, a0, a1);
            s.q0[i] = a0;
            s.q1[i] = a1;
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < sums; i += threads) {
        float a0 = 0.f, a1 = 0.f;
        if (shares > 1) {
#pragma unroll 8
            for (int j = 0; j < shares; ++j) { a0 += s.q0[j * sums + i]; a1 += s.q1[j * sums + i]; }
        } else for (int j = 0; j < terms; ++j) term(i, j, a0, a1);
        s.c0[i] = a0;
        s.c1[i] = a1;
        done(i, a0, a1);
    }
}

// the lanes' sums per channel: into LDS and, where wanted, to the parts
template <int V, bool FLAT, int GRAN>
__device__ __forceinline__ void channel_sums(const BackwardCall& f, const Lane<V, FLAT>& l, const Channels<V, FLAT, GRAN>& h, const SumSpace& s,
                                             const float (&s0)[V], const float (&s1)[V]) {
    const NormCall& c = f.n;
    const Tile& t = f.t;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        s.p0[threadIdx.x * V + i] = l.on ? s0[i] * c.drop.scale : 0.f;
        s.p1[threadIdx.x * V + i] = l.on ? s1[i] * (c.drop.scale * h.rstd[i / GRAN]) : 0.f;
    }
    __syncthreads();
    const int tc = t.channels, sums = t.units * tc, places = FLAT ? t.cols * V / tc : t.lane_rows, per_unit = t.cols * t.lane_rows * V;
    const uint32_t image0 = l.first_image, images = (uint32_t)(c.sets * c.images);
    add_up(s, sums, places,
           [&](int sum, int j, float& a0, float& a1) {
               const int unit = t.units > 1 ? sum / tc : 0, at = unit * per_unit + sum - unit * tc + j * tc;
               a0 += s.p0[at];
               a1 += s.p1[at];
           },
           [&](int sum, float a0, float a1) {
               const int unit = t.units > 1 ? sum / tc : 0, ch = (int)l.block * tc + sum - unit * tc;
               if (!f.parts || image0 + unit >= images || ch >= c.channels) return;
               float* to = f.parts + ((int64_t)(image0 + unit) * t.chunks + l.chunk) * 2 * c.channels + ch;
               to[0] = a0;
               to[c.channels] = a1;
           });
}

// A and B of the tile's groups from the channels' sums
template <int V, bool FLAT> __device__ __forceinline__ void group_means(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l, const SumSpace& s) {
    const int D = c.channels / c.groups, threads = blockDim.x, groups = t.units * t.groups, team = team_of(threads, groups, D), lane = threadIdx.x % team;
    const float n = (float)c.positions * (float)D;
    const uint32_t image0 = l.first_image, images = (uint32_t)(c.sets * c.images);
    for (int g = threadIdx.x / team; g < groups; g += threads / team) {
        const int unit = t.units > 1 ? g / t.groups : 0, in = (g - unit * t.groups) * D, ch0 = (int)l.block * t.channels + in;
        const uint32_t image = image0 + unit;
        float a0 = 0.f, a1 = 0.f;
        if (image < images && ch0 < c.channels) {
            for (int i = lane; i < D; i += team) {
                const int at = unit * t.channels + in + i;
                a0 += s.w[at] * s.c0[at];
                a1 += s.w[at] * s.c1[at];
            }
        }
        a0 = team_sum(a0, team);
        a1 = team_sum(a1, team);
        if (lane == 0) { s.g0[g] = a0 / n; s.g0[groups + g] = a1 / n; }
    }
}

// dx of pack k from dz (without scale) and x - m: r weight_c dz - ((x - m) r^2 B + r A).  (x r^2 B less a constant of the group m r^2 B would be an
// instruction per element less and 0 to 1.5 % faster, and off by m r 2^-24 of r B: a mean of ten thousand spreads in fp32, by 9e-4 of dx.)
template <class E, bool SILU, int V, bool FLAT, int GRAN>
__device__ __forceinline__ void write_dx(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l, const Channels<V, FLAT, GRAN>& h, const Place<V, FLAT>& to, int k,
                                         const float (&d)[V], float (&g)[V], const float (&rA)[V / GRAN], const float (&rrB)[V / GRAN]) {
    const float scale = c.drop.scale * (SILU ? SILU_BACK : 1.f);
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = __builtin_fmaf(g[i], h.w[i] * scale, -__builtin_fmaf(d[i], rrB[i / GRAN], rA[i / GRAN]));
    tile_store<E, V, FLAT>(t, l, (E*)c.out, to, k, packed<E, V>(g));
}

// Images that a workgroup holds: x and dy read once, x kept as it came and dz in fp32 from the sums to dx (a rounded dz would be another
// gradient, a second mask and sigmoid half the instructions again).  So four packs of bf16 per lane, 112 registers, two workgroups of 512 lanes per
// compute unit.  1024 images of 32x32x64 in bf16 with SiLU and dropout: 112 us, 3.6 TB/s of the 403 MB; 39 vector instructions per element keep
// the vector units busy for seven tenths of it, what is left is the two workgroups' waiting for loads and for each other's lanes.  In fp32
// with SiLU, 256 images of 28x28x40: 21.9 us, 4.4 TB/s (one workgroup per compute unit, and nothing to fill its waits).
template <class E, int V, int NV, bool FLAT, int GRAN, bool SILU, bool DROP>
__global__ void __launch_bounds__(1024) norm_backward_kernel(BackwardCall f) {
    constexpr int A = V / GRAN;
    extern __shared__ float lds[];
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t, tile_of_workgroup(gridDim.x));
    // (loads return in order: what the first pack needs is asked for before the packs)
    Channels<V, FLAT, GRAN> h(c, t, l);
    typename Pack<E, V>::type xv[NV], gv[NV];
    {
        const Place<V, FLAT> from(c, t, l, c.xs), at(c, t, l, c.dys);
        load_packs<NV>(t, l, 0, [&](int k, auto whole) {
            xv[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.x, from, f.x_extent, k);
            gv[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.dy, at, f.dy_extent, k);
        });
    }
    const SumSpace s(lds, blockDim.x * V, t.units * t.channels, t.units * t.groups, blockDim.x);
    h.share(t, l, s.w);
    h.template scale<SILU>();
    float dz[NV][V], s0[V], s1[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s0[i] = s1[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float d[V];
        h.template gradient<E, SILU, DROP>(c, k, xv[k], gv[k], d, dz[k]);
        add_pack<V, FLAT>(l.valid(t, k), d, dz[k], s0, s1);
#pragma unroll
        for (int i = 0; i < V; ++i) asm volatile("" : "+v"(dz[k][i]));      // (finished, and no select left for later)
        keep_packed(xv[k]);
        __builtin_amdgcn_sched_barrier(0);           // (a pack's registers at a time)
    }
    channel_sums(f, l, h, s, s0, s1);
    __syncthreads();
    group_means(c, t, l, s);
    __syncthreads();
    float rA[A], rrB[A];
#pragma unroll
    for (int a = 0; a < A; ++a) h.group_part(a, s.g0[l.unit * t.groups + h.group[a]], s.g0[(t.units + l.unit) * t.groups + h.group[a]], rA, rrB);
    const Place<V, FLAT> to(c, t, l, c.outs);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        float d[V];
        h.distances(xv[k], d);
        write_dx<E, SILU>(c, t, l, h, to, k, d, dz[k], rA, rrB);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Sums of a chunk per channel, in turns of GRAD_PACKS packs per lane, the next turn's on their way.  63 MB (x and dy of three images of
// 127x129x320 in bf16, SiLU) in 18.0 us, 3.5 TB/s.
template <class E, int V, bool FLAT, int GRAN, bool SILU, bool DROP>
__global__ void __launch_bounds__(512) norm_sums_kernel(BackwardCall f) {
    constexpr int NV = GRAD_PACKS;
    extern __shared__ float lds[];
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t, tile_of_workgroup(gridDim.x));
    const Place<V, FLAT> from(c, t, l, c.xs), at(c, t, l, c.dys);
    Channels<V, FLAT, GRAN> h(c, t, l);
    typename Pack<E, V>::type xn[NV], gn[NV];
    const auto packs_from = [&](int first) {
        load_packs<NV>(t, l, first, [&](int k, auto whole) {
            xn[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.x, from, f.x_extent, first + k);
            gn[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.dy, at, f.dy_extent, first + k);
        });
    };
    packs_from(0);
    h.template scale<SILU>();
    // SUM_RUN packs are added up one after the other, and so are their sums, which wait in the lane's place of the LDS
    const SumSpace s(lds, blockDim.x * V, t.channels, t.groups, blockDim.x);
    float *const before0 = s.p0 + threadIdx.x * V, *const before1 = s.p1 + threadIdx.x * V;
    float s0[V], s1[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s0[i] = s1[i] = 0.f;
    for (int turn = 0; turn < t.nv; turn += NV) {
        if (turn && turn % SUM_RUN == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                before0[i] = turn > SUM_RUN ? before0[i] + s0[i] : s0[i];
                before1[i] = turn > SUM_RUN ? before1[i] + s1[i] : s1[i];
                s0[i] = s1[i] = 0.f;
            }
        }
        typename Pack<E, V>::type xv[NV], gv[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) { xv[k] = xn[k]; gv[k] = gn[k]; }
        if (turn + NV < t.nv) packs_from(turn + NV);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float d[V], g[V];
            h.template gradient<E, SILU, DROP>(c, turn + k, xv[k], gv[k], d, g);
            add_pack<V, FLAT>(l.valid(t, turn + k), d, g, s0, s1);
        }
    }
    if (t.nv > SUM_RUN) {
#pragma unroll
        for (int i = 0; i < V; ++i) { s0[i] += before0[i]; s1[i] += before1[i]; }
    }
    channel_sums(f, l, h, s, s0, s1);
}

// dweight and dbias: a learner's sums over its images and their chunks.  A workgroup (the largest power of two of its lanes): `wide`
// channels (another), the rows dealt out to the lanes of a channel, then halves of these onto each other.  A lane's sum, of any
// number of terms, is kept in 64 bits (200000 vectors of 64, a constant gradient: in fp32 it is off by 1e-4), but eight of them are added first
// (20000 images of 6 positions, 33 channels in bf16, the whole backward pass: a 64-bit addition for each term 130 us, for eight 103).
__device__ __forceinline__ void add_parameters(const BackwardCall& f, uint32_t block, float* lds) {
    const NormCall& c = f.n;
    const int threads = 1 << (31 - __builtin_clz(blockDim.x)), wide = f.param_wide, lane = threadIdx.x;
    const uint32_t set = block / (uint32_t)f.param_blocks;
    const int ch = (int)(block - set * f.param_blocks) * wide + lane % wide, share = lane / wide, shares = threads / wide;
    const int64_t rows = c.images * f.chunks;
    double a = 0., b = 0.;
    if (lane < threads && ch < c.channels) {
        const float* p = f.parts + set * rows * 2 * c.channels + ch;
int64_t r = share;
        for (; r + 7 * shares < rows; r += 8 * shares) {
            float x[8], y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { const float* at = p + (r + i * shares) * 2 * c.channels; x[i] = at[0]; y[i] = at[c.channels]; }
            a += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            b += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
        }
        for (; r < rows; r += shares) { a += p[r * 2 * c.channels]; b += p[r * 2 * c.channels + c.channels]; }
    }
    if (lane < threads) { lds[lane] = (float)a; lds[threads + lane] = (float)b; }
    __syncthreads();
    for (int s = threads / 2; s >= wide; s /= 2) {
        if (lane < s) { lds[lane] += lds[lane + s]; lds[threads + lane] += lds[threads + lane + s]; }
        __syncthreads();
    }
    if (lane < wide && ch < c.channels) {
        if (c.dbias) c.dbias[set * c.dbias_stride + ch] = lds[lane];
        if (c.dweight) c.dweight[set * c.dweight_stride + ch] = lds[threads + lane];
    }
}

// dx of an image read again, by the workgroups that read the same tiles for the sums, on the same XCD and the last first: those are what
// its cache still holds.  Behind the tiles, the parameters.  Those 63 MB again and 31 MB written in 17.2 us, 5.5 TB/s.
template <class E, int V, bool FLAT, int GRAN, bool SILU, bool DROP>
__global__ void __launch_bounds__(512) norm_dx_kernel(BackwardCall f) {
    constexpr int A = V / GRAN, NV = GRAD_PACKS;
    extern __shared__ float lds[];
    if (blockIdx.x >= f.tiles) { add_parameters(f, blockIdx.x - f.tiles, lds); return; }
    const NormCall& c = f.n;
    const Tile& t = f.t;
    const Lane<V, FLAT> l(c, t, tile_of_workgroup(f.tiles, true));
    const Place<V, FLAT> from(c, t, l, c.xs), at(c, t, l, c.dys), to(c, t, l, c.outs);
    Channels<V, FLAT, GRAN> h(c, t, l);
    typename Pack<E, V>::type xn[NV], gn[NV];
    const auto packs_from = [&](int first) {
        load_packs<NV>(t, l, first, [&](int k, auto whole) {
            xn[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.x, from, f.x_extent, first + k);
            gn[k] = tile_load<E, V, FLAT, whole.value>(t, l, (const E*)c.dy, at, f.dy_extent, first + k);
        });
    };
    float rA[A], rrB[A];
    if (f.group_sums) {
        float gA[A], gB[A];
#pragma unroll
        for (int a = 0; a < A; ++a) { gA[a] = f.group_sums[2 * (h.first_group + h.group[a])]; gB[a] = f.group_sums[2 * (h.first_group + h.group[a]) + 1]; }
        packs_from(t.nv - NV);
        h.template scale<SILU>();
#pragma unroll
        for (int a = 0; a < A; ++a) h.group_part(a, gA[a], gB[a], rA, rrB);
    } else {
        // every workgroup adds up the chunks of its channels, JOINED_PARTS of them per lane at most
        const SumSpace s(lds, 0, t.channels, t.groups, blockDim.x);
        const int left = c.channels - (int)l.block * t.channels, sums = t.channels < left ? t.channels : left;
        const float* parts = f.parts + (int64_t)l.image * f.chunks * 2 * c.channels + l.block * t.channels;
        const int shares = shares_of(blockDim.x, t.channels, f.chunks), i = threadIdx.x;       // (t.channels * shares lanes at most)
        const int share = (int)((uint32_t)i / (uint32_t)t.channels), sum = i - share * t.channels;
        float p0[JOINED_PARTS], p1[JOINED_PARTS], a0 = 0.f, a1 = 0.f;
#pragma unroll
        for (int j = 0; j < JOINED_PARTS; ++j) {
            const int chunk = share + j * shares;
            const float* p = parts + (share < shares && chunk < f.chunks && sum < sums ? (int64_t)chunk * 2 * c.channels + sum : 0);
            p0[j] = p[0];
            p1[j] = p[c.channels];
        }
        packs_from(t.nv - NV);                               // (behind the parts, which come first)
        h.share(t, l, s.w);
        h.template scale<SILU>();
#pragma unroll
        for (int j = 0; j < JOINED_PARTS; ++j) if (share + j * shares < f.chunks) { a0 += p0[j]; a1 += p1[j]; }
        if (share < shares) { s.q0[i] = a0; s.q1[i] = a1; }
        __syncthreads();
        for (int i = threadIdx.x; i < t.channels; i += blockDim.x) {
            float a0 = 0.f, a1 = 0.f;
            for (int j = 0; j < shares; ++j) { a0 += s.q0[j * t.channels + i]; a1 += s.q1[j * t.channels + i]; }
            s.c0[i] = a0;
            s.c1[i] = a1;
        }
        __syncthreads();
        group_means(c, t, l, s);
        __syncthreads();
#pragma unroll
        for (int a = 0; a < A; ++a) h.group_part(a, s.g0[h.group[a]], s.g0[t.groups + h.group[a]], rA, rrB);
    }
    for (int turn = t.nv - NV; turn >= 0; turn -= NV) {
        typename Pack<E, V>::type xv[NV], gv[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) { xv[k] = xn[k]; gv[k] = gn[k]; }
        if (turn) packs_from(turn - NV);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float d[V], g[V];
            h.template gradient<E, SILU, DROP>(c, turn + k, xv[k], gv[k], d, g);
            write_dx<E, SILU>(c, t, l, h, to, turn + k, d, g, rA, rrB);
        }
    }
}

// A and B of a group from the sums of its image's chunks: a workgroup per group, a launch and its latency (4 to 5 us).
template <int T>
__global__ void __launch_bounds__(T) norm_group_kernel(BackwardCall f, float* group_sums) {
    __shared__ float lds[8];                         // (T = 256: four wavefronts)
    const NormCall& c = f.n;
    const uint32_t groups = (uint32_t)(c.sets * c.images * c.groups);
    for (uint32_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const uint32_t image = g / (uint32_t)c.groups, set = image / (uint32_t)c.images;
        const int D = c.channels / c.groups, first = (int)(g - image * c.groups) * D;
        const float* p = f.parts + (int64_t)image * f.chunks * 2 * c.channels + first;
        const float* w = c.weight ? c.weight + set * c.weight_stride + first : nullptr;
        double a = 0., b = 0.;                       // (chunks of any number)
        for (int r = threadIdx.x / D, i = threadIdx.x - r * D; r < f.chunks;) {
            const float wi = w ? w[i] : 1.f;
            a += wi * p[(int64_t)r * 2 * c.channels + i];
            b += wi * p[(int64_t)r * 2 * c.channels + c.channels + i];
            i += T;
            if (i >= D) { const int over = i / D; r += over; i -= over * D; }
        }
        const float wa = team_sum((float)a, 64), wb = team_sum((float)b, 64);
        if (threadIdx.x % 64 == 0) { lds[threadIdx.x / 64] = wa; lds[4 + threadIdx.x / 64] = wb; }
        __syncthreads();
        if (threadIdx.x < 2) {
            const float* q = lds + 4 * threadIdx.x;
            group_sums[2 * (int64_t)g + threadIdx.x] = ((q[0] + q[1]) + (q[2] + q[3])) / ((float)c.positions * (float)D);
        }
        __syncthreads();
    }
}

// The parameters' gradients behind norm_backward_kernel, whose sums per image it adds: a launch of its own, 4 to 5 us, for an order of the sums that
// does not depend on which workgroup ends first (atomics would).
template <int T>
__global__ void __launch_bounds__(T) norm_param_kernel(BackwardCall f) {
    extern __shared__ float lds[];
    const uint32_t blocks = (uint32_t)(f.n.sets * f.param_blocks);
    for (uint32_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        add_parameters(f, block, lds);
        __syncthreads();
    }
}

// ---- launches ----

// the tiles' workgroups and `more` behind them
template <class Kernel>
hipError_t start_backward(Kernel kernel, BackwardCall& f, size_t lds, int64_t more, hipStream_t st) {
    const Tile& t = f.t;
    const int64_t images = f.n.sets * f.n.images, tiles = (images + t.units - 1) / t.units * t.blocks * t.chunks;
    if ((tiles + more) * t.threads >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;
    if (lds > LDS_PLAIN) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    f.tiles = (uint32_t)tiles;
    kernel<<<dim3((unsigned)(tiles + more)), dim3(t.threads), lds, st>>>(f);
    return hipGetLastError();
}

// of a kernel that goes on with further work as long as there is some (a launch takes fewer than 2^32 lanes)
inline dim3 loop_grid(int64_t work) { return dim3((unsigned)(work < 1 << 20 ? work : 1 << 20)); }

// workgroups that add up the parameters' gradients
inline int64_t param_blocks(BackwardCall& f) {
    const NormCall& c = f.n;
    if (!c.dweight && !c.dbias) return 0;
    f.param_wide = 64;
    while (f.param_wide > 1 && f.param_wide / 2 >= c.channels) f.param_wide /= 2;
    f.param_blocks = (c.channels + f.param_wide - 1) / f.param_wide;
    return c.sets * f.param_blocks;
}

template <class E, int V, bool FLAT, int GRAN>
hipError_t backward_twice(BackwardCall& f, const NormTiles& t, float* workspace, hipStream_t st) {
    const NormCall& c = f.n;
    const int64_t images = c.sets * c.images, groups = images * c.groups;
    f.parts = workspace;
    f.chunks = t.sums.chunks;
    f.t = t.sums;
    return with_options(c, [&](auto silu, auto drop) {
        hipError_t e = start_backward(norm_sums_kernel<E, V, FLAT, GRAN, silu.value, drop.value>, f, f.t.lds, 0, st);
        if (e != hipSuccess) return e;
        // The workgroups that write dx add up the chunks of their channels themselves, where that is little beside their tile.
        if (t.apply.channels > t.apply.threads || f.chunks > JOINED_PARTS * shares_of(t.apply.threads, t.apply.channels, f.chunks)) {
            float* group_sums = workspace + images * f.chunks * 2 * c.channels;
            f.group_sums = group_sums;
            norm_group_kernel<256><<<loop_grid(groups), dim3(256), 0, st>>>(f, group_sums);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        f.t = t.apply;
        const int64_t params = param_blocks(f);
        const size_t space = (size_t)(2 * f.t.threads + 3 * f.t.channels + 2 * f.t.groups) * sizeof(float);
        return start_backward(norm_dx_kernel<E, V, FLAT, GRAN, silu.value, drop.value>, f, space, params, st);
    });
}

template <class E, int V, int NV, bool FLAT, int GRAN>
hipError_t backward_whole(BackwardCall& f, hipStream_t st) {
    return with_options(f.n, [&](auto silu, auto drop) {
        return start_backward(norm_backward_kernel<E, V, NV, FLAT, GRAN, silu.value, drop.value>, f, f.t.lds, 0, st);
    });
}

template <class E> hipError_t tiled_backward(const NormCall& c, const NormTiles& tiles, void* workspace, hipStream_t st) {
    BackwardCall f = {};
    f.n = c;
    f.x_extent = extent_of(c, c.xs);
    f.dy_extent = extent_of(c, c.dys);
    const bool whole = tiles.whole.nv != 0;
    f.t = whole ? tiles.whole : tiles.sums;
    return with_layout<E>(f.t, [&](auto vec, auto flat, auto gran) {
        constexpr int V = vec.value;
        constexpr int G = gran.value;
        constexpr bool FLAT = flat.value;
        if (!whole) return backward_twice<E, V, FLAT, G>(f, tiles, (float*)workspace, st);
        f.chunks = 1;
        const int64_t params = param_blocks(f);
        f.parts = params ? (float*)workspace : nullptr;
        hipError_t e;
        switch (f.t.nv) {
            case 1: e = backward_whole<E, V, 1, FLAT, G>(f, st); break;
            case 2: e = backward_whole<E, V, 2, FLAT, G>(f, st); break;
            case 4: e = backward_whole<E, V, backward_packs(G, V) < 4 ? backward_packs(G, V) : 4, FLAT, G>(f, st); break;
            default: e = backward_whole<E, V, backward_packs(G, V), FLAT, G>(f, st);
        }
        if (e != hipSuccess || !params) return e;
        norm_param_kernel<1024><<<loop_grid(params), dim3(1024), 2 * 1024 * sizeof(float), st>>>(f);
        return hipGetLastError();
    });
}

}  // namespace kavg
