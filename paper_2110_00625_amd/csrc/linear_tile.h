// Tiles of the products (linear.h) on the matrix cores: bf16 operands with v_mfma_f32_32x32x16_bf16, fp32 ones with v_mfma_f32_32x32x2_f32,
// sums in fp32.
//
// A workgroup owns a TR x TC tile of one learner's result, its WR x WC wavefronts MR x MC blocks of 32 x 32 of it each.  The contraction
// goes by slices of 128 bytes (BK = 64 or 32 elements), which lie in LDS in 16-byte chunks:
//   an operand whose contraction index is contiguous in memory as rows [x][128 bytes], chunk c of row x at c ^ (x/2 mod 8), so that the
//     sixteen lanes that read together find sixteen different banks' groups;
//   a turned operand as it lies in memory, [k][TX], its fragments taken by transposing reads (bf16) or single words (fp32); in bf16 the
//     chunks of row k are exchanged too, by blocks of four, with k mod 4 (rows of 256 bytes and more), so that four rows of a block of 32 lie in different banks.
// The lanes own slots of that layout in order, which is what loads from memory into LDS want; where an operand is not aligned to 16 bytes
// or its contiguous extent is no multiple of a chunk, a slice comes through registers into the same slots.  A slice is in flight while the one
// before it is multiplied (two LDS buffers), or three are, in a ring of four, where a compute unit has no more than two small tiles that could hide
// each other's latency.  Elements past the contraction are zeros; rows past an operand's extent are anything that can be read,
// they reach only results that are not stored.
//
// The matrix instruction's row index runs along c, so that a lane owns four consecutive columns of a row of the result.
//
// What bounds them.  Large tiles: 8192x4096x4096 in bf16 209 - 224 us by box (1.23 - 1.31 PFLOP/s; a library's product 180), its gradients 231 and 229 turned
// either way (248, 278); 8192x4096x16384 with SiLU and the pre-activation 927 - 970 (795 without them): the matrix cores are busy for 65 % of the
// cycles, at a clock that falls to 1.5 - 1.8 GHz under them; the rest are a pipeline's ends and results (100 us of the last) and waits for memory.  Steps on the
// way: the barrier in front of the last slab instead of the first and pinned orders 1190 -> 1044 (the gradient of x), waits that the compiler counts 227 -> 209,
// results through LDS 1085 -> 938.  In fp32 4096^3 takes 1010 us, 136 TFLOP/s of the 145 that a library's product reaches.  Small tiles: latency, 0.2 us a slice.
// Through registers: the wait for a whole slice in front of every barrier (four of 1001^3 in bf16 22 us, of 1000^3 straight into LDS 16; 3x1003x997x515 in fp32 43.6,
// the matrix cores busy for 45 % of the cycles).
// Tried: rings of slices of 64 bytes (half lines: 220 for 209, turned 282 for 239), four wavefronts of 128x128 (registers in scratch), tiles of 128x32,
// 32x128 and 128x64 (in no swept case better by more than 4 %).
#pragma once
#include "linear.h"
#include <type_traits>

namespace kavg {

struct ProductArgs {
    Matrix R, C;
    int nR, nC, nK;
    int tiles_r, tiles_c, splits, per_split;         // per_split: slices of a split
    uint32_t total, per_xcd;                         // workgroups, and of each of the 8 XCDs
    Finish finish;
    float* partial; int pitch; int64_t partial_split;    // or null: nothing is split
    int side; float* sums; int64_t sums_set, sums_split;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class E> struct Kind;
template <> struct Kind<__bf16> { typedef bf16x8 chunk; static constexpr int V = 8, BK = 64; };
template <> struct Kind<float> { typedef f32x4 chunk; static constexpr int V = 4, BK = 32; };
constexpr int SLICE_BYTES = 128, CHUNKS = 8;         // of a row

// which chunk of its row a slot holds
template <class E, int TX, bool TURNED> __device__ __forceinline__ int swizzle(int row) {
    if (!TURNED) return (row >> 1) & 7;
    return sizeof(E) == 2 && TX >= 128 ? (row & 3) * 4 : sizeof(E) == 2 && TX == 64 ? (row >> 1 & 1) * 4 : 0;
}

// Loads of one operand's slices; every lane owns N chunks of a slice.
template <class E, int TX, bool TURNED, int NT> struct Loader {
    static constexpr int V = Kind<E>::V, BK = Kind<E>::BK, N = TX * CHUNKS / NT, PER_ROW = TURNED ? TX / V : CHUNKS;
    static_assert(N * NT == TX * CHUNKS, "whole chunks per lane");
    const E* at[N];                 // of the present slice
    const E* end;                   // behind the operand's last element
    int k[N];                       // of the chunk's first element in a slice
    int x[N];                       // turned: of the chunk's first element
    int slot0;                      // of the wavefront's first chunk
    int64_t step, stride;

    __device__ __forceinline__ void init(const Matrix& m, int64_t set, int x0, int nX, int k0, int nK, int tid) {
        const E* base = (const E*)m.base + set * m.set_stride;
        stride = m.stride;
        step = TURNED ? BK * stride : BK;
        end = base + (TURNED ? (int64_t)(nK - 1) * stride + nX : (int64_t)(nX - 1) * stride + nK);
        slot0 = __builtin_amdgcn_readfirstlane(tid >> 6) * N * 64;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int slot = slot0 + i * 64 + (tid & 63), row = slot / PER_ROW, chunk = (slot % PER_ROW) ^ swizzle<E, TX, TURNED>(row);
            if (TURNED) {
                k[i] = row;
                x[i] = x0 + chunk * V < nX ? x0 + chunk * V : max(nX - V, 0);          // (past the extent: the last chunk)
                at[i] = base + (int64_t)(k0 + row) * stride + x[i];
            } else {
                k[i] = chunk * V;
                at[i] = base + (int64_t)min(x0 + row, nX - 1) * stride + k0 + k[i];
            }
        }
    }
    __device__ __forceinline__ void advance() {
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] += step;
    }
    // Straight into LDS; left: elements of the contraction from this slice on.  What lies past it (not WHOLE) is loaded from before its end, and
    // zeroed by fix() once it has landed.
    template <bool WHOLE> __device__ __forceinline__ void load(char* tile, int left) const {
        typedef __attribute__((address_space(3))) void* lds_p;
        typedef const __attribute__((address_space(1))) void* glb_p;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const E* p = at[i];
            if (!WHOLE) {
                const int over = TURNED ? k[i] - left + 1 : k[i] + V - left;
                if (over > 0) p -= TURNED ? over * stride : (int64_t)over;
            }
            __builtin_amdgcn_global_load_lds((glb_p)p, (lds_p)(tile + (slot0 + i * 64) * 16), 16, 0, 0);
        }
    }
    __device__ __forceinline__ void fix(char* tile, int left, int tid) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (k[i] >= left) *(u32x4*)(tile + (slot0 + i * 64 + (tid & 63)) * 16) = (u32x4){0u, 0u, 0u, 0u};
    }
    // Through registers, at any alignment and length.  (A turned operand's last chunk of a row may be read into what follows, as far as the operand
    // reaches in memory.)
    __device__ __forceinline__ void fetch(u32x4 (&r)[N], int left, int nX) const {
        if (TURNED ? left > BK && stride >= V && nX >= V : left >= BK) {             // (another row follows the slice's; all of its chunks are there)
#pragma unroll
            for (int i = 0; i < N; ++i) r[i] = __builtin_bit_cast(u32x4, pack_load<E, V>(at[i]));
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int there = TURNED ? nX - x[i] : left - k[i];
            const int whole = !TURNED ? there : k[i] >= left ? 0 : there > 0 && end - at[i] >= V ? V : there;
            if (whole >= V) r[i] = __builtin_bit_cast(u32x4, pack_load<E, V>(at[i]));
            else {
                typename Kind<E>::chunk c;
#pragma unroll
                for (int e = 0; e < V; ++e) c[e] = e < whole ? at[i][e] : (E)0.f;
                r[i] = __builtin_bit_cast(u32x4, c);
            }
        }
    }
    __device__ __forceinline__ void put(const u32x4 (&r)[N], char* tile, int tid) const {
#pragma unroll
        for (int i = 0; i < N; ++i) *(u32x4*)(tile + (slot0 + i * 64 + (tid & 63)) * 16) = r[i];
    }
};

// The operand of a matrix instruction: slab kk (two chunks) of the 32 rows from x0 on.
template <class E, int TX, bool TURNED> __device__ __forceinline__ typename Kind<E>::chunk fragment(const char* tile, int x0, int kk, int lane) {
    const int half = lane >> 5;
    if constexpr (!TURNED) {
        const int x = x0 + (lane & 31);
        return *(const typename Kind<E>::chunk*)(tile + x * SLICE_BYTES + ((kk * 2 + half) ^ swizzle<E, TX, false>(x)) * 16);
    } else if constexpr (sizeof(E) == 2) {
        // in a group of 16 lanes, lane 4a + b fetches x = 4b .. 4b+3 of row a and receives the four rows of x = 4a + b
        const int t = lane & 15, group = lane >> 4, row = kk * 16 + (group >> 1) * 8 + (t >> 2);
        const int chunk = (x0 / 8 + (group & 1) * 2 + ((t & 3) >> 1)) ^ swizzle<E, TX, true>(row);
        const char* p = tile + row * (TX * 2) + chunk * 16 + (t & 1) * 8;
        typedef bf16x4 __attribute__((address_space(3))) * lds_ptr;
        const char* q = tile + (row + 4) * (TX * 2) + ((x0 / 8 + (group & 1) * 2 + ((t & 3) >> 1)) ^ swizzle<E, TX, true>(row + 4)) * 16 + (t & 1) * 8;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_ptr)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_ptr)q);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        f32x4 v;
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = *(const float*)(tile + (kk * 8 + half * 4 + t) * (TX * 4) + (x0 + (lane & 31)) * 4);
        return v;
    }
}

__device__ __forceinline__ f32x16 multiply(const bf16x8& c, const bf16x8& r, f32x16 acc) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(c, r, acc, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(const f32x4& c, const f32x4& r, f32x16 acc) {
    // (element t of both chunks: k = t of the lower lanes' chunk and of the upper lanes')
#pragma unroll
    for (int t = 0; t < 4; ++t) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(c[t], r[t], acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ void add_up(const bf16x8& f, float (&s)[4]) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_fdot2_f32_bf16((pair){f[2 * i], f[2 * i + 1]}, ones, s[i], false);
}
__device__ __forceinline__ void add_up(const f32x4& f, float (&s)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += f[i];
}

template <class E, int TR, int TC, int WR, int WC, int BUFFERS, bool RT, bool CT, bool DIRECT> struct ProductTile {
    static constexpr int NT = 64 * WR * WC, MR = TR / (32 * WR), MC = TC / (32 * WC);
    static constexpr int BUFFER = (TR + TC) * SLICE_BYTES;
    static constexpr int PITCH = MC * 32 + 4, STAGE = WR * WC * 32 * PITCH * 4;            // rows of results on their way out
    static constexpr int RING = DIRECT ? BUFFERS : 2, LDS = RING * BUFFER > STAGE ? RING * BUFFER : STAGE;
};

template <class E, int TR, int TC, int WR, int WC, int BUFFERS, bool RT, bool CT, bool DIRECT>
__global__ void __launch_bounds__(64 * WR * WC) product_kernel(ProductArgs a) {
    typedef ProductTile<E, TR, TC, WR, WC, BUFFERS, RT, CT, DIRECT> P;
    typedef typename Kind<E>::chunk chunk;
    constexpr int NT = P::NT, MR = P::MR, MC = P::MC, BK = Kind<E>::BK, SLABS = 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WC, wc = wave % WC;

    // Workgroups go round the 8 XCDs in launch order; each XCD takes a run of tiles, which share operands in its L2, eight rows of tiles at a time.
    const uint32_t number = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
    if (number >= a.total) return;
    const uint32_t tiles = (uint32_t)a.tiles_r * a.tiles_c, which = number / tiles, tile = number - which * tiles;
    const int64_t set = which / (uint32_t)a.splits;
    const int split = (int)(which % (uint32_t)a.splits);
    const uint32_t band = tile / (8u * a.tiles_c), in_band = tile - band * 8u * a.tiles_c, height = min(8u, (uint32_t)a.tiles_r - band * 8u);
    const int tile_c = (int)(in_band / height), tile_r = (int)(band * 8 + in_band % height);
    const int r0 = tile_r * TR, c0 = tile_c * TC;
    const int slice0 = split * a.per_split, slices = min(a.per_split, (a.nK + BK - 1) / BK - slice0);
    int left = a.nK - slice0 * BK;

    Loader<E, TR, RT, NT> rl;
    Loader<E, TC, CT, NT> cl;
    rl.init(a.R, set, r0, a.nR, slice0 * BK, a.nK, tid);
    cl.init(a.C, set, c0, a.nC, slice0 * BK, a.nK, tid);

    f32x16 acc[MR][MC];
#pragma unroll
    for (int i = 0; i < MR; ++i)
#pragma unroll
        for (int j = 0; j < MC; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    constexpr int MS = MR > MC ? MR : MC;
    float sums[RT ? MS : 1][4] = {};
    double totals[RT ? MS : 1] = {};
    const bool sum_r = RT && a.side == 1 && tile_c == 0 && wc == 0, sum_c = RT && a.side == 2 && tile_r == 0 && wr == 0;

    // Sums of dz: a run of 2048 rows in fp32 (256 terms to each of a lane's four), runs in 64 bits, so that any number of rows will do.
    constexpr int RUN = 2048 / BK;
    auto end_run = [&](int slices_done) {
        if (!RT || slices_done % RUN || !(sum_r || sum_c)) return;
#pragma unroll
        for (int i = 0; i < (RT ? MS : 1); ++i) {
            totals[i] += (double)((sums[i][0] + sums[i][1]) + (sums[i][2] + sums[i][3]));
            sums[i][0] = sums[i][1] = sums[i][2] = sums[i][3] = 0.f;
        }
    };

    // Fragments of a slab are asked for while the one before it is multiplied: two sets of registers.
    chunk rf[2][MR], cf[2][MC];
    auto take = [&](int to, const char* buffer, int slab) {
#pragma unroll
        for (int j = 0; j < MC; ++j) cf[to][j] = fragment<E, TC, CT>(buffer + TR * SLICE_BYTES, (wc * MC + j) * 32, slab, lane);
#pragma unroll
        for (int i = 0; i < MR; ++i) rf[to][i] = fragment<E, TR, RT>(buffer, (wr * MR + i) * 32, slab, lane);
    };
    auto multiply_slab = [&](int from) {
#pragma unroll
        for (int i = 0; i < MR; ++i)
#pragma unroll
            for (int j = 0; j < MC; ++j) acc[i][j] = multiply(cf[from][j], rf[from][i], acc[i][j]);
        if (sum_r) {
#pragma unroll
            for (int i = 0; i < MR; ++i) add_up(rf[from][i], sums[RT ? i : 0]);
        }
        if (sum_c) {
#pragma unroll
            for (int j = 0; j < MC; ++j) add_up(cf[from][j], sums[RT ? j : 0]);
        }
    };

    // The order for the scheduler (which would fold the two sets into one): an LDS read or two behind every product, and loads of a slice as many.
    auto interleave = [&](auto loads) {
        constexpr int READS = MC * (!CT ? 1 : sizeof(E) == 2 ? 2 : 4) + MR * (!RT ? 1 : sizeof(E) == 2 ? 2 : 4), PRODUCTS = MR * MC * (sizeof(E) == 2 ? 1 : 4);
        constexpr int LOADS_EACH = 2;
        constexpr int EACH = READS <= 2 * PRODUCTS ? 2 : (READS + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i * EACH < READS) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
            else if (loads.value) __builtin_amdgcn_sched_group_barrier(0x020, LOADS_EACH, 0);
        }
    };

    if constexpr (DIRECT) {
        // The barrier of a slice lies before its last slab is multiplied: by then every wavefront has that slab in registers, so that the buffer takes
        // the slice after the next, and the next slice's first slab is read under those products.
        constexpr int LOADS = rl.N + cl.N;
        auto load = [&](auto whole, char* to, int rest) {
            rl.template load<whole.value>(to, rest);
            cl.template load<whole.value>(to + TR * SLICE_BYTES, rest);
            rl.advance();
            cl.advance();
        };
        auto mend = [&](char* slice, int rest) {
            if (rest < BK) {
                rl.fix(slice, rest, tid);
                cl.fix(slice + TR * SLICE_BYTES, rest, tid);
            }
        };
        constexpr std::true_type whole = {};
        constexpr std::false_type cut = {};
        // Waits as the compiler counts them (it would add its own behind an asm's), with no access to memory moved across.
        constexpr int RING = P::RING, FLYING = LOADS * (RING - 2), FIRST = FLYING + LOADS;
        static_assert(FIRST < 64, "the wait counter");
        auto wait = [&](auto counts) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(counts.value);
            asm volatile("" ::: "memory");
        };
        auto meet = [&] {
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        // vmcnt n, bits 3:0 and 15:14; expcnt 7; lgkmcnt, bits 11:8, 15 (any) or 0
        constexpr std::integral_constant<int, (FIRST & 15) | (FIRST >> 4) << 14 | 0x0F70> first_landed = {};
        constexpr std::integral_constant<int, (FLYING & 15) | (FLYING >> 4) << 14 | 0x0070> next_landed_and_read = {};
        constexpr std::integral_constant<int, 0x0F70> all_landed = {};
        constexpr std::integral_constant<int, 0xC07F> lds_done = {};
#pragma unroll
        for (int i = 0; i < RING; ++i) if (i < slices) load(cut, lds + i * P::BUFFER, left - i * BK);
        if (slices >= RING) wait(first_landed);
        else wait(all_landed);
        mend(lds, left);
        wait(lds_done);
        meet();
        take(0, lds, 0);
        char *now = lds, *next = lds + P::BUFFER;
        auto first_slabs = [&] {
#pragma unroll
            for (int slab = 0; slab + 1 < SLABS; ++slab) {
                take(~slab & 1, now, slab + 1);
                multiply_slab(slab & 1);
                interleave(std::integral_constant<int, 0>());
            }
        };
        auto turn = [&] {
            now = next;
            next = next == lds + (RING - 1) * P::BUFFER ? lds : next + P::BUFFER;
        };
        int s = 0;
        for (const int full = min(left / BK, slices); s + RING < full; ++s, left -= BK) {   // the slices that this loop loads are whole ones
            first_slabs();
            __builtin_amdgcn_sched_barrier(0);               // (no product of theirs behind the barrier, where it would wait for the others)
            wait(next_landed_and_read);                      // (this wavefront's part of the next slice, its reads of this one)
            meet();
            take(0, next, 0);
            load(whole, now, left);
            multiply_slab((SLABS - 1) & 1);
            interleave(std::integral_constant<int, LOADS>());
            end_run(s + 1);
            turn();
        }
        for (; s < slices; ++s, left -= BK) {
            first_slabs();
            if (s + 1 < slices) {
                wait(all_landed);
                mend(next, left - BK);
                wait(lds_done);
                meet();
                take(0, next, 0);
                if (s + RING < slices) load(cut, now, left - RING * BK);
            }
            multiply_slab((SLABS - 1) & 1);
            turn();
        }
    } else {
        u32x4 rr[rl.N], cr[cl.N];
        rl.fetch(rr, left, a.nR);
        cl.fetch(cr, left, a.nC);
        for (int s = 0; s < slices; ++s, left -= BK) {
            char* now = lds + (s & 1) * P::BUFFER;
            rl.put(rr, now, tid);
            cl.put(cr, now + TR * SLICE_BYTES, tid);
            __syncthreads();                                 // (the buffer's last reads lie before the last barrier)
            if (s + 1 < slices) {
                rl.advance();
                cl.advance();
                rl.fetch(rr, left - BK, a.nR);
                cl.fetch(cr, left - BK, a.nC);
            }
            take(0, now, 0);
#pragma unroll
            for (int slab = 0; slab < SLABS; ++slab) {
                if (slab + 1 < SLABS) take(~slab & 1, now, slab + 1);
                multiply_slab(slab & 1);
            }
            end_run(s + 1);
        }
    }

    if (RT && (sum_r || sum_c)) {
        float* to = a.sums + set * a.sums_set + split * a.sums_split;
        const int first = sum_r ? r0 + wr * MR * 32 : c0 + wc * MC * 32, n = sum_r ? a.nR : a.nC;
#pragma unroll
        for (int i = 0; i < MS; ++i) {
            if (i >= (sum_r ? MR : MC)) break;
            const double half = totals[RT ? i : 0] + (double)((sums[RT ? i : 0][0] + sums[RT ? i : 0][1]) + (sums[RT ? i : 0][2] + sums[RT ? i : 0][3]));
            const float sum = (float)(half + __shfl_xor(half, 32));
            const int x = first + i * 32 + lane;
            if (lane < 32 && x < n) to[x] = sum;
        }
    }
    // Results leave through LDS, by wavefront: 32 rows of its columns at a time, so that the lanes of a row write whole lines (and the code is there once
    // for eight columns of a lane, not for every register).  The hardware keeps a wavefront's accesses to LDS in order; the fences keep the compiler, to which a
    // lane's reads are of other places than its writes, from exchanging them.
    constexpr int WTC = MC * 32, PITCH = P::PITCH, ROW_LANES = WTC / 8, ROWS = 64 / ROW_LANES, TURNS = 32 / ROWS;
    __syncthreads();
    float* stage = (float*)lds + wave * 32 * PITCH;
    const int first = c0 + wc * WTC, down = lane / ROW_LANES;
    auto emit = [&](const auto& finish, auto apart) {
        const int col = (lane % ROW_LANES) * (apart.value == 4 ? 8 : 4);
#pragma unroll
        for (int i = 0; i < MR; ++i) {
#pragma unroll
            for (int j = 0; j < MC; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) *(f32x4*)(stage + (lane & 31) * PITCH + j * 32 + q * 8 + (lane >> 5) * 4) = (f32x4){acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
            finish(r0 + (wr * MR + i) * 32 + down, ROWS, a.nR, [&](int u, float (&v)[8]) {
                const float* from = stage + (down + u * ROWS) * PITCH + col;
                const f32x4 lo = *(const f32x4*)from, hi = *(const f32x4*)(from + apart.value);
#pragma unroll
                for (int k = 0; k < 4; ++k) { v[k] = lo[k]; v[4 + k] = hi[k]; }
            });
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        }
    };
    typedef typename std::conditional<RT, float, E>::type O;
    constexpr int FAR = WTC / 2, APART = sizeof(O) == 4 ? FAR : 4;
    const int c = first + (lane % ROW_LANES) * (APART == 4 ? 8 : 4);
    const std::integral_constant<int, APART> apart = {};
    if (a.partial) {
        Finish parts = {};
        parts.floor = -INFINITY;
        parts.out = a.partial + split * a.partial_split; parts.out_set = (int64_t)a.nR * a.pitch; parts.out_row = a.pitch;
        const int c = first + (lane % ROW_LANES) * 4;
        emit(Finisher<E, float, TURNS, false, FAR>(parts, set, c, a.pitch - c), std::integral_constant<int, FAR>());       // (rows are padded to whole eights)
    } else if (c0 + TC <= a.nC) emit(Finisher<E, O, TURNS, true, APART>(a.finish, set, c, 0), apart);
    else emit(Finisher<E, O, TURNS, false, APART>(a.finish, set, c, a.nC - c), apart);
}

// Tiles: rows, columns, wavefronts along rows and columns, buffers.  The last is that of few small tiles with a long contraction, in bf16.
#define KAVG_TILES(TILE) TILE(0, 256, 256, 2, 4, 2) TILE(1, 128, 128, 2, 2, 2) TILE(2, 64, 64, 2, 2, 2) TILE(3, 64, 64, 2, 2, 4)
enum { TILE_LARGE = 0, TILE_MIDDLE = 1, TILE_SMALL = 2, TILE_DEEP = 3, TILE_KINDS = 4 };

// DIRECT wants operands whose chunks are aligned and whole; the first and the last tile are for such operands only, the last
// for bf16 operands that are not turned
template <class E, int TR, int TC, int WR, int WC, int BUFFERS, bool RT, bool CT, bool DIRECT>
hipError_t start_tile(const ProductArgs& a, hipStream_t st) {
    typedef ProductTile<E, TR, TC, WR, WC, BUFFERS, RT, CT, DIRECT> P;
    const auto kernel = product_kernel<E, TR, TC, WR, WC, BUFFERS, RT, CT, DIRECT>;
    if (P::LDS > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
        if (e != hipSuccess) return e;
    }
    kernel<<<dim3(8 * a.per_xcd), dim3(P::NT), P::LDS, st>>>(a);
    return hipGetLastError();
}

template <class E, bool RT, bool CT> hipError_t start_kind(int tile, bool direct, const ProductArgs& a, hipStream_t st) {
#define TILE(NUMBER, TR, TC, WR, WC, BUFFERS) \
    case NUMBER: \
        if constexpr (BUFFERS == 2 || (!CT && sizeof(E) == 2)) { if (direct) return start_tile<E, TR, TC, WR, WC, BUFFERS, RT, CT, true>(a, st); } \
        if constexpr (TR * TC < 256 * 256 && BUFFERS == 2) return start_tile<E, TR, TC, WR, WC, BUFFERS, RT, CT, false>(a, st); \
        break;
    switch (tile) { KAVG_TILES(TILE) }
#undef TILE
    return hipErrorInvalidValue;
}

}  // namespace kavg
