// Group norm in tiles that stay in registers: what the forward and the backward kernels share.
//
// A tile is some channels (whole groups) of a run of an image's positions.  A lane owns packs of V elements (16 bytes, or 8 of
// bf16; one element where no pack fits), NV of them: always the same V channels, at positions `lane_rows` apart, so that parameters and sums of a channel
// stay in the lane's registers, and a wavefront reads and writes whole segments of rows.
//
//   rows   V divides the channels: a row is a position, a pack never leaves it.
//   flat   V does not, but the positions of an image lie end to end: the image is one run of elements, cut into rows of `cols` packs.
//          cols * V is a multiple of the channels, so a lane's packs still hold the same channels (going round after the last one).
//   V = 1  neither.
//
// An image that one workgroup cannot hold is read twice: first for its sums, by workgroups that go through a chunk of it in turns, then
// for its results.  Small images share a workgroup (units).
#pragma once
#include "layers.h"
#include <type_traits>

namespace kavg {

struct Tile {
    int nv, vec;             // packs per lane, elements per pack
    bool flat;
    int gran;                // elements of a pack that always lie in one group (a power of two)
    int threads, units;      // lanes of a workgroup, images of a workgroup
    int cols, lane_rows;     // packs per row, rows that the lanes of a unit cover together
    int channels, groups;    // of a tile
    int blocks, chunks;      // tiles of an image: along its channels, along its rows
    int rows, whole_rows;    // of an image; rounds of the lanes (flat: rows) that it fills
    // divisions by lanes per unit, cols, channels per group, sums of a row per group (packs, or channels)
    // tiles along the rows and the channels, images of a learner
    Divisor by_unit, by_cols, by_d, by_per, by_chunks, by_blocks, by_images;
    size_t lds;
};

// Tiles of a call: one for a workgroup that holds its part of an image (whole.nv > 0), or two, for sums and for results.
struct NormTiles { Tile whole, sums, apply; };

constexpr int FORWARD_PACKS = 16;  // the most packs per lane
constexpr int FLAT_PACKS = 8;      // of a flat tile (its sums are per channel, and its last pack needs care: more spill)
// of the backward pass, which holds x and dz (in fp32) of each
constexpr int backward_packs(int gran, int vec) { return vec == 8 ? gran == 1 ? 2 : 4 : 8; }
constexpr int SUM_PACKS = 4;       // of a turn of the forward sums, which holds two turns
constexpr int GRAD_PACKS = 2;      // of a turn of the backward sums
constexpr int APPLY_PACKS = 4;
constexpr int SUM_RUN = 128;       // packs of the backward sums that are added up in one go (a chunk of 1 MB; images of 4 GB and more have some thousand)

constexpr int JOINED_PARTS = 4;    // chunks per lane that the workgroups of the results join themselves
constexpr size_t LDS_PLAIN = 64 * 1024;      // more than that has to be asked for

// elements of a tensor from its first to its last
inline int64_t extent_of(const NormCall& c, const Strides& s) {
    return (c.sets - 1) * s.set + (c.images - 1) * s.image + (c.positions - 1) * s.row + c.channels;
}

// false: no tile fits (groups too wide for a workgroup)
bool norm_tiles(const NormCall& c, bool contiguous, bool backward, NormTiles* t);
// The same of a call with its operands: flat only where the positions of each lie end to end and what is read holds a pack at least.  (A pack
// at the end of a tensor is moved to end with it, see tile_load; images that share memory make a tensor shorter than its elements are many.)
bool call_tiles(const NormCall& c, bool backward, NormTiles* t);
size_t norm_workspace(const NormCall& c, const NormTiles& t, bool backward);
// values of a group in a whole chunk, in positions
inline int64_t chunk_positions(const NormCall& c, const Tile& t) { return (int64_t)t.nv * (t.flat ? (int64_t)t.cols * t.vec / c.channels : t.lane_rows); }

// lanes that add up `terms` terms each of `sums` sums together: a power of two, at most a wavefront
KAVG_FD int team_of(int threads, int sums, int terms) {
    int team = 64;
    while (team > 1 && (team / 2 >= terms || threads / team < sums)) team /= 2;
    return team;
}

template <class E> hipError_t tiled_forward(const NormCall& c, const NormTiles& t, void* workspace, hipStream_t st);
template <class E> hipError_t tiled_backward(const NormCall& c, const NormTiles& t, void* workspace, hipStream_t st);

// f(constants: elements of a pack, flat, elements of it in one group) of a tile
template <int V, class F> hipError_t with_granules(const Tile& t, F f) {
    constexpr std::integral_constant<int, V> pack = {};
    if (t.gran == V) return f(pack, std::false_type(), pack);
    if (t.gran == V / 2) return f(pack, std::false_type(), std::integral_constant<int, V / 2>());
    return t.gran == 2 ? f(pack, std::false_type(), std::integral_constant<int, 2>()) : f(pack, std::false_type(), std::integral_constant<int, 1>());
}
template <class E, class F> hipError_t with_layout(const Tile& t, F f) {
    constexpr int V = 16 / (int)sizeof(E);
    constexpr std::integral_constant<int, 1> one = {};
    if (t.vec == 1) return f(one, std::false_type(), one);
    if (t.flat) return f(std::integral_constant<int, V>(), std::true_type(), one);
    return t.vec == V ? with_granules<V>(t, f) : with_granules<4>(t, f);
}
// f(constants: SiLU, dropout)
template <class F> hipError_t with_options(const NormCall& c, F f) {
    if (c.drop.threshold) return c.silu ? f(std::true_type(), std::true_type()) : f(std::false_type(), std::true_type());
    return c.silu ? f(std::true_type(), std::false_type()) : f(std::false_type(), std::false_type());
}

#if defined(__HIPCC__)

// Workgroup g runs on XCD g mod 8, and tiles next to each other share lines of memory and parameters, so each XCD takes a contiguous range
// of them.  backwards: its range from the end.
__device__ __forceinline__ uint32_t tile_of_workgroup(uint32_t tiles, bool backwards = false) {
    const uint32_t per = tiles / 8, extra = tiles % 8, x = blockIdx.x % 8, at = blockIdx.x / 8;
    return x * per + (x < extra ? x : extra) + (backwards ? per + (x < extra) - 1 - at : at);
}

// v, worked out in scalar registers (what follows would be moved in front of the choice that led here, into vector registers)
__device__ __forceinline__ int64_t scalar(int64_t v) { asm volatile("" : "+s"(v)); return v; }

// Where a lane works.  What all lanes share (everything but unit, row and col where a workgroup has one image) is worked out in scalar
// registers: in the vector ones these few 64-bit products were a seventh of the backward pass's instructions.
template <int V, bool FLAT> struct Lane {
    uint32_t unit, row, col;                        // row, col: in the unit
    bool in;                                        // the lane has a place in a unit
    uint32_t chunk, block;                          // of the tile
    uint32_t first_image, first_set, first_in_set;  // of the tile: number of all learners', learner, number of the learner's
    uint32_t image, set, image_in_set;              // of the lane's unit
    int first_channel;                              // of the lane's pack (flat: within the image's channels)
    bool on;                                        // the place has an image and channels
    int64_t run;                                    // elements of an image

    __device__ __forceinline__ Lane(const NormCall& c, const Tile& t, uint32_t tile) {
        unit = t.units > 1 ? divide(threadIdx.x, t.by_unit) : 0;
        uint32_t at = threadIdx.x - unit * (t.cols * t.lane_rows);
        in = unit < (uint32_t)t.units && at < (uint32_t)(t.cols * t.lane_rows);
        if (!in) unit = at = 0;
        row = FLAT ? 0 : divide(at, t.by_cols);
        col = at - row * t.cols;
        run = (int64_t)c.positions * c.channels;
        const uint32_t rest = divide(tile, t.by_chunks);
        chunk = tile - rest * t.chunks;
        const uint32_t first = divide(rest, t.by_blocks);
        block = rest - first * t.blocks;
        first_image = first * t.units;
        first_set = divide(first_image, t.by_images);
        first_in_set = first_image - first_set * (uint32_t)c.images;
        on = in;
        image = first_image;
        set = first_set;
        image_in_set = first_in_set;
        if (t.units > 1) {
            on = in && first_image + unit < (uint32_t)(c.sets * c.images);
            if (on) image += unit;
            set = divide(image, t.by_images);
            image_in_set = image - set * (uint32_t)c.images;
        }
        if (FLAT) first_channel = (int)(col * V % (uint32_t)c.channels);
        else {
            first_channel = block * t.channels + col * V;
            if (first_channel >= c.channels) { on = false; first_channel = 0; }
        }
    }
    __device__ __forceinline__ void channels(const NormCall& c, int (&ch)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) ch[i] = first_channel + i;
        if (!FLAT) return;
        if (V <= c.channels) {
#pragma unroll
            for (int i = 1; i < V; ++i) ch[i] -= ch[i] >= c.channels ? c.channels : 0;
        } else {
            for (int i = 1; i < V; ++i) ch[i] %= c.channels;
        }
    }
    // where the lane's image, its learner's parameters, the tile's groups (a lane without work: groups that exist) and the first element of
    // the image's number lie
    __device__ __forceinline__ int64_t image_at(const Tile& t, const Strides& s) const {
        if (t.units > 1) return set * s.set + image_in_set * s.image;
        return scalar(first_set * s.set + first_in_set * s.image);
    }
    __device__ __forceinline__ int64_t set_at(const Tile& t, int64_t stride) const {
        if (t.units > 1) return set * stride;
        return scalar(first_set * stride);
    }
    __device__ __forceinline__ int64_t groups_at(const NormCall& c, const Tile& t) const {
        if (t.units > 1) return (int64_t)image * c.groups + block * t.groups;
        return scalar((int64_t)first_image * c.groups + block * t.groups);
    }
    __device__ __forceinline__ uint64_t number_of_image(const Tile& t) const {
        if (t.units > 1) return (uint64_t)image * run;
        return scalar((int64_t)first_image * run);
    }
    // row of the image of lane 0's pack k, and of the lane's
    __device__ __forceinline__ int first_row(const Tile& t, int k) const { return (int)(chunk * t.nv + k) * t.lane_rows; }
    __device__ __forceinline__ int image_row(const Tile& t, int k) const { return first_row(t, k) + (int)row; }
    // is every lane's pack k one of the image's?  (The same in all lanes.)
    __device__ __forceinline__ bool whole(const Tile& t, int k) const { return (int)(chunk * t.nv + k) < t.whole_rows; }
    // elements of pack k that are the image's
    __device__ __forceinline__ int valid(const Tile& t, int k) const {
        const int r = image_row(t, k);
        if (!FLAT) return on && r < t.rows ? V : 0;
        if (whole(t, k)) return on ? V : 0;
        uint32_t at = col;
        asm volatile("" : "+v"(at));                // (asked again, worked out again: answers per pack and element would fill the scalar registers)
        const int64_t left = run - ((int64_t)r * t.cols + at) * V;
        return !on || left <= 0 ? 0 : left < V ? (int)left : V;
    }
    // number of pack 0's first element in the whole tensor; what a pack more adds
    __device__ __forceinline__ uint64_t number(const NormCall& c, const Tile& t) const {
        const int64_t before = scalar((int64_t)first_row(t, 0) * (FLAT ? t.cols * V : c.channels));
        return number_of_image(t) + before + (FLAT ? col * V : (uint64_t)row * (uint32_t)c.channels + first_channel);
    }
    __device__ __forceinline__ uint64_t number_step(const NormCall& c, const Tile& t) const {
        return FLAT ? (uint64_t)t.cols * V : (uint64_t)t.lane_rows * c.channels;
    }
};

// A lane's packs in a tensor: from `first` on, `step` apart.
template <int V, bool FLAT> struct Place {
    int64_t first, step;
    __device__ __forceinline__ Place(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l, const Strides& s) {
        const int64_t image = l.image_at(t, s);
        step = FLAT ? (int64_t)t.cols * V : t.lane_rows * s.row;
        first = image + scalar(l.first_row(t, 0) * (FLAT ? step : s.row)) + (FLAT ? l.col * V : (int64_t)((uint64_t)l.row * (uint64_t)s.row) + l.first_channel);
        // (a lane without a pack 0 reads the image's first row)
        if (!l.whole(t, 0) && !l.valid(t, 0)) first = image + (FLAT ? 0 : l.first_channel);
    }
};

// of the chunk: rows (flat: elements) of a round of the lanes, whole rounds, and rows of the last one; its positions
template <int V, bool FLAT> struct Chunk {
    int64_t step;
    int rounds, rest;
    float positions;
    __device__ __forceinline__ Chunk(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l) {
        step = FLAT ? (int64_t)t.cols * V : t.lane_rows;
        const int64_t all = (FLAT ? l.run : t.rows) - (int64_t)l.chunk * t.nv * step, here = all < t.nv * step ? all : t.nv * step;
        rounds = (int)((uint32_t)(here / step));
        rest = (int)(here - rounds * step);
        positions = (float)(FLAT ? here / c.channels : here);
    }
    // rounds in which a place of the lanes (row; flat: element) is the image's
    __device__ __forceinline__ int rounds_of(int place) const { return rounds + (place < rest); }
};

// Pack k of a tensor; pack 0 once more where the image has no such pack.  One at a flat image's end may reach past it, into the next image,
// which does no harm, but not past the tensor (extent): there it is put together from single elements.  No load but those stands behind
// a branch that lanes take apart.
template <class E, int V, bool FLAT, bool WHOLE>
__device__ __forceinline__ typename Pack<E, V>::type tile_load(const Tile& t, const Lane<V, FLAT>& l, const E* p, const Place<V, FLAT>& at0, int64_t extent, int k) {
    if (WHOLE) return pack_load<E, V>(p + at0.first + k * at0.step);
    int64_t at = at0.first + (l.valid(t, k) ? k * at0.step : 0);
    asm("" : "+v"(at));                              // (or the compiler makes that a copy of pack 0, behind a branch and a wait for it)
    if (!FLAT) return pack_load<E, V>(p + at);
    typename Pack<E, V>::type v = pack_load<E, V>(p + (at + V <= extent ? at : extent - V));
    if (at + V > extent) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = at + i < extent ? p[at + i] : (E)0.f;
    }
    return v;
}

// load(k, is it whole?) of the lane's packs first .. first+NV-1; in rows all of them in one branch or the other
template <int NV, int V, bool FLAT, class F> __device__ __forceinline__ void load_packs(const Tile& t, const Lane<V, FLAT>& l, int first, F load) {
    if (FLAT) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (l.whole(t, first + k)) load(k, std::true_type());
            else load(k, std::false_type());
        }
    } else if (l.whole(t, first + NV - 1)) {
#pragma unroll
        for (int k = 0; k < NV; ++k) load(k, std::true_type());
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) load(k, std::false_type());
    }
}

template <class E, int V> __device__ __forceinline__ typename Pack<E, V>::type packed(const float (&v)[V]) {
    typename Pack<E, V>::type o;
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {             // (two at a time, so that they are converted together)
            const typename Pack<float, 2>::type two = {v[i], v[i + 1]};
            const typename Pack<E, 2>::type r = __builtin_convertvector(two, typename Pack<E, 2>::type);
            o[i] = r[0];
            o[i + 1] = r[1];
        }
    } else o[0] = from_float<E>(v[0]);
    return o;
}

template <class E, int V, bool FLAT>
__device__ __forceinline__ void tile_store(const Tile& t, const Lane<V, FLAT>& l, E* p, const Place<V, FLAT>& at0, int k, const typename Pack<E, V>::type& o) {
    const int n = l.valid(t, k);
    if (!n) return;
    p += at0.first + k * at0.step;
    if (!FLAT || n == V) pack_store<E, V>(p, o);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) if (i < n) p[i] = o[i];
    }
}

// A learner's parameters of the lane's channels, or in their place one number for all of them: no load behind a branch (a wait for it would
// follow, in front of the packs').
static __device__ float no_weight[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}, no_bias[8] = {};      // (never written; not const, for constants
                                                                                                    // lie in another kind of memory)
template <int V, bool FLAT>
__device__ __forceinline__ void lane_parameters(const Lane<V, FLAT>& l, const int (&ch)[V], const float* of, int64_t at, const float* none, float (&p)[V]) {
    const float* from = of ? of + at : none;
    const int each = of ? -1 : 0;
    if (FLAT) {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = from[ch[i] & each];
    } else {
        constexpr int N = V < 4 ? V : 4;
        from += l.first_channel & each;
#pragma unroll
        for (int i = 0; i < V; i += N) {
            const typename Pack<float, N>::type v = pack_load<float, N>(from + i);
#pragma unroll
            for (int j = 0; j < N; ++j) p[i + j] = v[j];
        }
    }
}
// the channels' weights and biases, and the groups in the tile of the lane's A sums (of a lane without work, whose group may not exist: the first)
template <int V, bool FLAT, int A>
__device__ __forceinline__ void lane_parameters(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l, float (&w)[V], float (&b)[V], int (&group)[A]) {
    int ch[V];
    l.channels(c, ch);
    lane_parameters(l, ch, c.weight, l.set_at(t, c.weight_stride), no_weight, w);
    lane_parameters(l, ch, c.bias, l.set_at(t, c.bias_stride), no_bias, b);
#pragma unroll
    for (int a = 0; a < A; ++a) group[a] = l.on ? divide(FLAT ? ch[a] : l.col * V + a * (V / A), t.by_d) : 0;
}

// bf16 packs stay packed between their uses (the compiler would keep their floats, twice the registers).
template <class P> __device__ __forceinline__ void keep_packed(P& v) {
    if constexpr (sizeof(P) >= 8 && sizeof(v[0]) == 2) {
        typedef int words __attribute__((ext_vector_type(sizeof(P) / 4)));
        words w = __builtin_bit_cast(words, v);
        asm volatile("" : "+v"(w));
        v = __builtin_bit_cast(P, w);
    }
}

// The lane's masks: a pack more is a whole number of draws further (V = 4, 8: the elements between two packs are a multiple of V), so that a
// pack's state is an addition away.  Packs begin with a draw but in flat images that are not made of draws.
template <int V, bool FLAT> struct TileMask {
    uint64_t first, step;                           // V > 1: states of draws, else numbers of elements
    uint32_t phase;
    bool aligned;
    __device__ __forceinline__ TileMask(const NormCall& c, const Tile& t, const Lane<V, FLAT>& l) {
        const uint64_t e = l.number(c, t), each = l.number_step(c, t);
        const DropPlace at(c.drop, e);
        first = V > 1 ? at.state : e;
        step = V > 1 ? each / 4 * SPLITMIX_GAMMA : each;
        phase = at.phase;
        aligned = !FLAT || l.run % 4 == 0;
    }
    // of pack k
    template <class E> __device__ __forceinline__ void drop(const DropRule& d, int k, typename Pack<E, V>::type& v) const {
        if constexpr (V == 1) v[0] = drop_keeps(d, first + k * step) ? v[0] : (E)0.f;
        else if (aligned) drop_pack<E, V, true>(d, DropPlace(first + k * step, 0), v);
        else drop_pack<E, V, false>(d, DropPlace(first + k * step, phase), v);
    }
};

// sum + N elements of a pack from the first-th on, in bf16 two at a time (exact products with one, fp32 sums)
template <int N, class P> __device__ __forceinline__ float pack_sum(const P& v, int first, float sum) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    if constexpr (sizeof(v[0]) == 2 && N > 1) {
        const pair ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
        for (int i = 0; i < N; i += 2) { const pair p = {v[first + i], v[first + i + 1]}; sum = __builtin_amdgcn_fdot2_f32_bf16(p, ones, sum, false); }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) sum += to_float(v[first + i]);
    }
    return sum;
}

// the same of squares (bf16)
template <int N, class P> __device__ __forceinline__ float pack_squares(const P& v, int first, float sum) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < N; i += 2) { const pair p = {v[first + i], v[first + i + 1]}; sum = __builtin_amdgcn_fdot2_f32_bf16(p, p, sum, false); }
    return sum;
}

__device__ __forceinline__ float team_sum(float v, int team) {
    for (int m = team / 2; m; m /= 2) v += __shfl_xor(v, m);
    return v;
}
#endif

}  // namespace kavg
