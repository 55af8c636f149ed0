// Products of few rows, or of few outputs (up to 16), whose operands' contraction lies together: answers for single samples, last layers.  The weights (or
// the many rows) are read once, for two flops a row and 2 or 4 bytes: bound by memory.  A workgroup owns 16 or 32 outputs of a learner; its eight wavefronts
// go through the contraction in turns of 128 bytes of every weight row, straight from memory into the operands of matrix instructions of 16 x 16 (a
// lane's two chunks are its share of the turn: any order of the contraction will do, as long as both operands have it), and their sums meet in
// LDS, in order.  No LDS in the loop, no split contraction, one launch.
// A call in a graph: 1 row of 4096x4096 in bf16 7.4 us (4.5 TB/s, 2.5 of it the launch's), 11 rows 9.2, 16 rows in fp32 18.0, 16 learners' 128x1024x10 in fp32
// 5.9; through tiles, split and joined, 9.5, 9.5, 26 and 10.8.  Tried: rounds in two sets of registers, one loaded while the other is multiplied (4 rows of
// 4096x16384 30.3 for 26.8: fewer wavefronts), a ring of turns in registers (30.3), loads of whole lines, eight rows' turns at a time (8.2 and 32: twice
// the products and sums), sixteen wavefronts (18.6 in fp32, the same in bf16), 17 to 32 rows in two blocks (13.8: x is read as often as the weights).
#include "linear_tile.h"

namespace kavg {

namespace {

constexpr int WAVES = 8, AT_ONCE = 4;

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 multiply16(const bf16x8& c, const bf16x8& r, f32x4 acc) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, r, acc, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply16(const f32x4& c, const f32x4& r, f32x4 acc) {
#pragma unroll
    for (int t = 0; t < 4; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(c[t], r[t], acc, 0, 0, 0);
    return acc;
}

// CB: blocks of 16 outputs.  Rows and outputs past the last are read as the last and not stored.  TURNED: a product of few outputs instead, a last layer's;
// rows and outputs change places until the results are stored.
template <class E, int CB, bool TURNED>
__global__ void __launch_bounds__(64 * WAVES) rows_kernel(ProductArgs a) {
    typedef typename Kind<E>::chunk chunk;
    constexpr int V = Kind<E>::V, TURN = 8 * V, ROUND = AT_ONCE * WAVES * TURN, PITCH = CB * 16 + 4;
    __shared__ float parts[WAVES][16][PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t set = blockIdx.x / (uint32_t)a.tiles_c;
    const int c0 = (int)(blockIdx.x - set * a.tiles_c) * CB * 16, k0 = wave * TURN + (lane >> 4) * V;
    const Matrix &C = TURNED ? a.R : a.C, &R = TURNED ? a.C : a.R;
    const int nC = TURNED ? a.nR : a.nC, nR = TURNED ? a.nC : a.nR;
    const E* cp[CB];
#pragma unroll
    for (int j = 0; j < CB; ++j) cp[j] = (const E*)C.base + set * C.set_stride + min(c0 + j * 16 + (lane & 15), nC - 1) * C.stride;
    const E* rp = (const E*)R.base + set * R.set_stride + min(lane & 15, nR - 1) * R.stride;
    f32x4 acc[CB];
#pragma unroll
    for (int j = 0; j < CB; ++j) acc[j] = (f32x4){0.f, 0.f, 0.f, 0.f};

    // a round: four turns of every wavefront, all asked for before the first is multiplied
    auto some = [&](auto whole, int k) {
        chunk c[AT_ONCE][2][CB], r[AT_ONCE][2];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = k + u * WAVES * TURN + h * 4 * V;
                const bool there = whole.value || at < a.nK;             // (whole chunks)
#pragma unroll
                for (int j = 0; j < CB; ++j) c[u][h][j] = there ? *(const chunk*)(cp[j] + at) : (chunk)0.f;
                r[u][h] = there ? *(const chunk*)(rp + at) : (chunk)0.f;
            }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < CB; ++j) acc[j] = multiply16(c[u][h][j], r[u][h], acc[j]);
    };
    int done = 0;
    for (; done + ROUND <= a.nK; done += ROUND) some(std::true_type(), done + k0);
    if (done < a.nK) some(std::false_type(), done + k0);

#pragma unroll
    for (int j = 0; j < CB; ++j) *(f32x4*)&parts[wave][lane & 15][j * 16 + (lane >> 4) * 4] = acc[j];
    __syncthreads();
    const int lanes = TURNED ? 2 : 2 * CB, row = threadIdx.x / lanes, col = threadIdx.x % lanes * 8;        // of the tile, as it is stored
    if (row >= (TURNED ? CB * 16 : 16)) return;
    const int r = TURNED ? c0 + row : row, c = TURNED ? col : c0 + col;
    const Finisher<E, E, 1, false> finish(a.finish, set, c, a.nC - c);
    finish(r, 1, a.nR, [&](int, float (&v)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += TURNED ? parts[w][col + k][row] : parts[w][row][col + k];
    });
}

template <class E, int CB, bool TURNED> hipError_t start(ProductArgs a, int64_t sets, hipStream_t st) {
    a.tiles_c = ((TURNED ? a.nR : a.nC) + CB * 16 - 1) / (CB * 16);
    rows_kernel<E, CB, TURNED><<<dim3((unsigned)(sets * a.tiles_c)), dim3(64 * WAVES), 0, st>>>(a);
    return hipGetLastError();
}

template <class E, bool TURNED> hipError_t start(const ProductArgs& a, int64_t sets, hipStream_t st) {
    // twice as many outputs per read of x where even so every compute unit has two workgroups
    return sets * (((TURNED ? a.nR : a.nC) + 31) / 32) >= 512 ? start<E, 2, TURNED>(a, sets, st) : start<E, 1, TURNED>(a, sets, st);
}

}  // namespace

hipError_t start_rows(int dtype, const ProductArgs& a, int64_t sets, hipStream_t st) {
    return dtype == KAVG_BF16 ? start<__bf16, false>(a, sets, st) : start<float, false>(a, sets, st);
}
hipError_t start_columns(int dtype, const ProductArgs& a, int64_t sets, hipStream_t st) {
    return dtype == KAVG_BF16 ? start<__bf16, true>(a, sets, st) : start<float, true>(a, sets, st);
}

}  // namespace kavg
