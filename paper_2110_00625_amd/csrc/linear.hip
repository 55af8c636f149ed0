// Products of learners' layers: which tile a call takes, whether its contraction is split, and the launch that joins the parts.
#include "linear_tile.h"
#include <algorithm>

namespace kavg {

hipError_t start_rows(int dtype, const ProductArgs& a, int64_t sets, hipStream_t st);
hipError_t start_columns(int dtype, const ProductArgs& a, int64_t sets, hipStream_t st);
hipError_t start_bf16_plain(int tile, bool direct, const ProductArgs& a, hipStream_t st);
hipError_t start_bf16_turned(int tile, bool direct, const ProductArgs& a, hipStream_t st);
hipError_t start_bf16_gradient(int tile, bool direct, const ProductArgs& a, hipStream_t st);
hipError_t start_f32_plain(int tile, bool direct, const ProductArgs& a, hipStream_t st);
hipError_t start_f32_turned(int tile, bool direct, const ProductArgs& a, hipStream_t st);
hipError_t start_f32_gradient(int tile, bool direct, const ProductArgs& a, hipStream_t st);

namespace {

constexpr int CUS = 256;
constexpr int T = 256;
constexpr int MOST_ROWS = 16;                    // that the kernel of few rows takes
constexpr int64_t MOST_ELEMENTS = 1 << 25;       // of weights in bf16, there
constexpr int64_t MOST_TILES = 1 << 22;          // of a launch (fewer than 2^32 lanes)

struct Size { int r, c; };
constexpr Size tile_size(int tile) {
#define TILE(NUMBER, TR, TC, WR, WC, BUFFERS) if (tile == NUMBER) return {TR, TC};
    KAVG_TILES(TILE)
#undef TILE
    return {0, 0};
}

// elements of a slice of the contraction
int slice_of(int dtype) { return dtype == KAVG_BF16 ? Kind<__bf16>::BK : Kind<float>::BK; }

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

int64_t tiles_of(int tile, int64_t sets, int nR, int nC) {
    const Size s = tile_size(tile);
    return sets * up(nR, s.r) * std::max<int64_t>(1, up(nC, s.c));
}

// The sum of n parts by G lanes that follow each other: each adds up every G-th, eight of which are asked for at a time, then they add in a tree.
template <int V, int G> __device__ __forceinline__ void add_parts(const float* p, int64_t apart, int n, int lane, float (&v)[V]) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = 0.f;
    for (int s = lane % G; s < n; s += 8 * G) {
        float t[8][V];
#pragma unroll
        for (int u = 0; u < 8; ++u) load_some<float, V>(p + min(s + u * G, n - 1) * apart, V, t[u]);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s + u * G < n) {
#pragma unroll
                for (int k = 0; k < V; ++k) v[k] += t[u][k];
            }
    }
#pragma unroll
    for (int d = 1; d < G; d *= 2)
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] += __shfl_xor(v[k], d);
}

// Sums of an operand of a weight gradient: [split][set][x] and where they go.
struct SumsArgs { const float* parts; float* sums; int64_t split, from_set, to_set, n, sets; };

// G lanes add up the parts of eight columns of a row and the first finishes them; the workgroups behind the last row's add up the operand's sums.
template <class E, int G>
__global__ void __launch_bounds__(T) join_kernel(ProductArgs a, uint64_t packs, uint32_t groups, uint32_t per_row, Divisor by_row, SumsArgs sums) {
    constexpr int EACH = T / G;                             // packs of a workgroup
    const int lane = threadIdx.x, own = lane / G;
    if (blockIdx.x >= groups) {
        const int64_t i = min((int64_t)(blockIdx.x - groups) * EACH + own, sums.sets * sums.n - 1), set = i / sums.n, x = i - set * sums.n;
        float v[1];
        add_parts<1, G>(sums.parts + set * sums.from_set + x, sums.split, a.splits, lane, v);
        sums.sums[set * sums.to_set + x] = v[0];            // (lanes past the last have the last)
        return;
    }
    const uint64_t first = (uint64_t)blockIdx.x * EACH;
    // (a row has fewer than 2^28 packs, so that what is divided stays below 2^30)
    const uint64_t row0 = first / per_row, last = packs - 1 - first;
    const uint32_t at = (uint32_t)(first - row0 * per_row) + (uint32_t)min((uint64_t)own, last), down = divide(at, by_row);
    const uint64_t row = row0 + down;
    const int c = (int)(at - down * per_row) * 8;
    float v[8];
    add_parts<8, G>(a.partial + row * a.pitch + c, a.partial_split, a.splits, lane, v);
    if ((uint64_t)own > last || lane % G) return;
    const int64_t set = (int64_t)(row / (uint64_t)a.nR), r = (int64_t)(row - (uint64_t)set * a.nR);
    const Finisher<E, E, 1, false> finish(a.finish, set, c, a.nC - c);
    finish(r, 1, a.nR, [&](int, float (&to)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) to[k] = v[k];
    });
}
// (eight lanes for a pack where there are few packs and parts for each lane: 8 results of 64x64 of 32 parts 7.2 us and 5.3)
template <class E> hipError_t start_join(const ProductArgs& a, uint64_t packs, const SumsArgs& sums, hipStream_t st) {
    const uint32_t per_row = (uint32_t)a.pitch / 8;
    const Divisor by_row = divisor(std::max<uint32_t>(per_row, 1));
    const int lanes = a.splits >= 8 && packs <= 64 * 1024 ? 8 : 1, each = T / lanes;
    const uint32_t groups = (uint32_t)up(packs, each);
    const dim3 grid(groups + (uint32_t)up(sums.n * sums.sets, each));
    if (lanes == 8) join_kernel<E, 8><<<grid, dim3(T), 0, st>>>(a, packs, groups, per_row, by_row, sums);
    else join_kernel<E, 1><<<grid, dim3(T), 0, st>>>(a, packs, groups, per_row, by_row, sums);
    return hipGetLastError();
}

bool aligned(const Matrix& m, int64_t sets, int64_t lines, int extent, int elem) {
    const int chunk = 16 / elem;
    return !((uintptr_t)m.base & 15) && extent % chunk == 0 && (sets < 2 || m.set_stride % chunk == 0) && (lines < 2 || m.stride % chunk == 0);
}

}  // namespace

// What a tile of each kind costs, in microseconds: a slice of 128 bytes where a compute unit has one tile of them, and per tile where it has more;
// filling and emptying the pipeline.  (256 compute units; 8192x4096x4096 in bf16 by large tiles 234 us, middle 260, small 376, four products of 1000^3 by
// large, split in two, 33, middle 16, small 20, 2048x1024x1024 by middle 12, small 9; 1024x8192x1024 by middle 37, split in eight 32, deep 30; 4096^3 in
// fp32 by large 1032, middle 1004, small 1106.)
struct Cost { float alone, shared, ends; };
static constexpr Cost BF16_COST[TILE_KINDS] = {{1.75f, 1.75f, 8.f}, {0.5f, 0.48f, 2.f}, {0.24f, 0.17f, 0.5f}, {0.21f, 0.15f, 0.8f}};
static constexpr Cost F32_COST[TILE_DEEP] = {{8.f, 8.f, 8.f}, {1.95f, 1.95f, 2.f}, {0.52f, 0.52f, 0.5f}};

Plan product_plan(int dtype, int64_t sets, int nR, int nC, int nK, Turned turned) {
    const int64_t slices = up(nK, slice_of(dtype));
    Plan p = {};
    p.pitch = (int)up(nC, 8) * 8;
    p.splits = 1;
    float least = INFINITY;
    for (int tile = 0; tile < TILE_KINDS; ++tile) {
        // (turned operands gain nothing by slices further ahead: 16 learners' 128x1024x1024 10.5 us by deep tiles and 11.7 by small ones, turned 13.6 and 13.0; fp32
        // ones neither, whose products take longer than the loads)
        if (tile == TILE_DEEP && (dtype != KAVG_BF16 || turned != NONE_TURNED)) break;
        const Cost& c = (dtype == KAVG_BF16 ? BF16_COST : F32_COST)[tile];
        const int64_t tiles = tiles_of(tile, sets, nR, nC);
        for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (splits > 1 && (2 * splits > slices || tiles * splits > 8 * CUS)) break;
            const int64_t each = up(slices, splits), m = up(tiles * up(slices, std::max<int64_t>(each, 1)), CUS);
            if (tile == TILE_DEEP && m > 2) continue;
            float cost = m * c.ends + each * std::max(c.alone, c.shared * m);
            // the launch that joins the parts, which are written and read
            if (splits > 1) cost += 4.f + 0.1f * splits + (float)sets * nR * p.pitch * splits * 8 / 5.5e6f;
            if (cost < least) { least = cost; p.tile = tile; p.splits = (int)std::max<int64_t>(1, up(slices, std::max<int64_t>(each, 1))); }
        }
    }
    if (p.splits > 1) p.bytes = (size_t)p.splits * sets * ((size_t)nR * p.pitch + (turned == BOTH_TURNED ? std::max(nR, nC) : 0)) * sizeof(float);
    return p;
}

namespace {

enum class Way { ROWS, COLUMNS, TILES };
struct Course { Way way; bool direct; Plan plan; };

// Which kernel a product takes.
Course course_of(const ProductCall& call) {
    const bool bf16 = call.dtype == KAVG_BF16;
    const int elem = bf16 ? 2 : 4;
    Course c = {Way::TILES, false, {}};
    c.direct = call.nC && call.nK && aligned(call.R, call.sets, call.r_turned ? call.nK : call.nR, call.r_turned ? call.nR : call.nK, elem) &&
               aligned(call.C, call.sets, call.c_turned ? call.nK : call.nC, call.c_turned ? call.nC : call.nK, elem);
    if (c.direct && !call.r_turned && !call.c_turned) {
        // Larger matrices in bf16 come faster through tiles, whose loads never pause (4 rows of 4096x4096 7.5 us and 9.5 through tiles, of 4096x8192 15.6 and
        // 15.5, of 4096x16384 27.6 and 21.2; 16 rows of 4096x4096 in fp32 17 and 26, which its products take).
        auto fits = [&](int64_t lines) { return call.sets * up(lines, 16) <= MOST_TILES && (!bf16 || call.sets * lines * call.nK <= MOST_ELEMENTS); };
        if (call.nR <= MOST_ROWS && fits(call.nC)) c.way = Way::ROWS;
        // (every wavefront has a part of the contraction)
        else if (call.nC <= MOST_ROWS && call.nK >= 8 * slice_of(call.dtype) && fits(call.nR)) c.way = Way::COLUMNS;
    }
    if (c.way == Way::TILES)
        c.plan = product_plan(call.dtype, call.sets, call.nR, call.nC, call.nK, call.r_turned ? BOTH_TURNED : call.c_turned ? C_TURNED : NONE_TURNED);
    return c;
}

hipError_t workspace_ok(const Plan& plan, const void* workspace, size_t bytes) {
    if (plan.splits < 2) return hipSuccess;
    if (bytes < plan.bytes) return hipErrorOutOfMemory;
    return !workspace || ((uintptr_t)workspace & 15) ? hipErrorInvalidValue : hipSuccess;
}

}  // namespace

hipError_t check_product(const ProductCall& call, const void* workspace, size_t bytes) {
    return workspace_ok(course_of(call).plan, workspace, bytes);
}

hipError_t launch_product(const ProductCall& call, void* workspace, size_t bytes, hipStream_t st) {
    const bool bf16 = call.dtype == KAVG_BF16;
    const int elem = bf16 ? 2 : 4;
    const Course course = course_of(call);
    if (course.way != Way::TILES) {
        ProductArgs a = {};
        a.R = call.R; a.C = call.C;
        a.nR = call.nR; a.nC = call.nC; a.nK = call.nK;
        a.finish = call.finish;
        return course.way == Way::ROWS ? start_rows(call.dtype, a, call.sets, st) : start_columns(call.dtype, a, call.sets, st);
    }
    const Plan& plan = course.plan;
    const bool direct = course.direct;
    const hipError_t fits = workspace_ok(plan, workspace, bytes);
    if (fits != hipSuccess) return fits;
    const int tile = direct ? plan.tile : plan.tile == TILE_LARGE ? TILE_MIDDLE : plan.tile == TILE_DEEP ? TILE_SMALL : plan.tile;
    const Size size = tile_size(tile);

    ProductArgs a = {};
    a.nC = call.nC; a.nK = call.nK;
    a.tiles_c = (int)std::max<int64_t>(1, up(call.nC, size.c));
    a.splits = plan.splits;
    a.per_split = (int)up(up(call.nK, slice_of(call.dtype)), plan.splits);
    a.finish = call.finish;
    a.side = call.side;
    a.sums = call.sums; a.sums_set = call.sums_set;
    // as many learners and rows at once as a launch takes (all of them, but for more than four million learners of small layers or hundreds of millions of rows)
    const int64_t of_row = (int64_t)a.tiles_c * a.splits, rows_at_once = std::min<int64_t>(call.nR, std::max<int64_t>(1, MOST_TILES / of_row) * size.r);
    const int64_t sets_at_once = rows_at_once < call.nR ? 1 : std::max<int64_t>(1, MOST_TILES / (of_row * up(call.nR, size.r)));
    if (of_row > MOST_TILES || (plan.splits > 1 && (rows_at_once < call.nR || sets_at_once < call.sets))) return hipErrorInvalidValue;
    for (int64_t set = 0; set < call.sets; set += sets_at_once)
        for (int64_t r = 0; r < call.nR; r += rows_at_once) {
            const int64_t sets = std::min(sets_at_once, call.sets - set);
            auto moved = [&](const void* p, int64_t elements, int size) { return p ? (void*)((char*)p + elements * size) : nullptr; };
            a.nR = (int)std::min(rows_at_once, call.nR - r);
            a.R = call.R; a.C = call.C;
            a.R.base = moved(call.R.base, set * call.R.set_stride + (call.r_turned ? r : r * call.R.stride), elem);
            a.C.base = moved(call.C.base, set * call.C.set_stride, elem);
            Finish& f = a.finish;
            f.bias = (const float*)moved(call.finish.bias, set * f.bias_set, 4);
            f.kept = moved(call.finish.kept, set * f.kept_set + r * f.kept_row, elem);
            f.before = moved(call.finish.before, set * f.before_set + r * f.before_row, elem);
            f.residual = moved(call.finish.residual, set * f.residual_set + r * f.residual_row, elem);
            f.out = moved(call.finish.out, set * f.out_set + r * f.out_row, call.r_turned ? 4 : elem);
            if (call.side) a.sums = call.sums + set * call.sums_set + (call.side == 1 ? r : 0);
            a.tiles_r = (int)up(a.nR, size.r);
            a.total = (uint32_t)(sets * a.splits * a.tiles_r * a.tiles_c);
            a.per_xcd = (uint32_t)up(a.total, 8);
            SumsArgs sums = {};
            if (plan.splits > 1) {
                a.partial = (float*)workspace;
                a.pitch = plan.pitch;
                a.partial_split = sets * (int64_t)a.nR * a.pitch;
                if (call.side) {
                    const int64_t n = call.side == 1 ? a.nR : a.nC;
                    sums = {a.partial + plan.splits * a.partial_split, a.sums, sets * n, n, call.sums_set, n, sets};
                    a.sums = (float*)sums.parts; a.sums_set = n; a.sums_split = sums.split;
                }
            }
            const auto start = call.r_turned ? (bf16 ? start_bf16_gradient : start_f32_gradient)
                                             : call.c_turned ? (bf16 ? start_bf16_turned : start_f32_turned) : (bf16 ? start_bf16_plain : start_f32_plain);
            hipError_t e = start(tile, direct, a, st);
            if (e != hipSuccess) return e;
            if (plan.splits > 1) {
                const uint64_t packs = (uint64_t)sets * a.nR * (plan.pitch / 8);
                e = bf16 && !call.r_turned ? start_join<__bf16>(a, packs, sums, st) : start_join<float>(a, packs, sums, st);
                if (e != hipSuccess) return e;
            }
        }
    return hipSuccess;
}

}  // namespace kavg
