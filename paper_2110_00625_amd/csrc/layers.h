// Launch interface of the layers (kavg_group_norm, kavg_dropout) and what their kernels share.  The boundary (layers_api.hip) has
// checked every argument; launchers derive grids.
#pragma once
#include "kavg_internal.h"
#include "counter_stream.h"
#include "fastdiv.h"

namespace kavg {

// which elements are dropped, and by what the others are multiplied
struct DropRule {
    uint64_t base;        // seed + (1 + site 2^40) gamma
    uint32_t threshold;   // 0: none is dropped; 65536: all
    float scale;
};
DropRule drop_rule(double drop, uint64_t seed, uint64_t site);

// Division of n < 2^30 (fastdiv.h) in 32-bit steps: n itself for m = 0, else the upper half of n m, shifted
struct Divisor { uint32_t m; int shift; };
inline Divisor divisor(uint32_t d) {
    Divisor v = {0, 0};
    if (d > 1) { fastdiv_make(d, &v.m, &v.shift); v.shift -= 32; }
    return v;
}

struct Strides { int64_t set, image, row; };

struct NormCall {
    int dtype;
    bool silu;                              // else ReLU above `floor` (see activate)
    float floor;
    int64_t sets, images, positions;
    int channels, groups;
    float eps;
    DropRule drop;
    const void* x; Strides xs;
    const void* dy; Strides dys;            // backward
    void* out; Strides outs;                // y, or dx
    const float* weight; int64_t weight_stride;
    const float* bias; int64_t bias_stride;
    float* mean; float* rstd;               // written by the forward pass (or null), read by the backward pass
    float* dweight; int64_t dweight_stride; // backward, or null
    float* dbias; int64_t dbias_stride;
};

size_t norm_workspace(const NormCall& c, bool backward);
// hipErrorOutOfMemory, hipErrorInvalidValue: a workspace too small, misaligned or not there, before anything is launched
hipError_t launch_group_norm(const NormCall& c, void* workspace, size_t bytes, hipStream_t st);
hipError_t launch_group_norm_backward(const NormCall& c, void* workspace, size_t bytes, hipStream_t st);

struct DropCall {
    int dtype;
    const void* x; int64_t x_stride;
    const void* residual; int64_t residual_stride;   // or null
    void* y; int64_t y_stride;
    int64_t rows, cols;
    DropRule drop;
};
hipError_t launch_dropout(const DropCall& c, hipStream_t st);

#if defined(__HIPCC__)
__device__ __forceinline__ uint32_t divide(uint32_t n, Divisor d) { return d.m ? __umulhi(n, d.m) >> d.shift : n; }

// 64 bits for the four elements 4q .. 4q+3
__device__ __forceinline__ uint64_t drop_bits(const DropRule& d, uint64_t q) { return splitmix64_mix(d.base + q * SPLITMIX_GAMMA); }
__device__ __forceinline__ bool drop_keeps(const DropRule& d, uint64_t e) {
    const uint64_t word = drop_bits(d, e >> 2);
    uint32_t upper = (uint32_t)(word >> 32);
    asm("" : "+v"(upper));                       // (a choice of halves, not a 64-bit shift: see drop_pack)
    const uint32_t half = e & 2 ? upper : (uint32_t)word;
    return (half >> (16 * ((uint32_t)e & 1)) & 0xFFFF) >= d.threshold;
}

// V consecutive elements in registers and in memory, at any multiple of an element's size (the hardware takes 16-byte accesses at any
// address; one that straddles a line costs a second one)
template <class E, int V> struct Pack {
    typedef E type __attribute__((ext_vector_type(V)));
    typedef type loose __attribute__((aligned(sizeof(E))));
};
template <class E, int V> __device__ __forceinline__ typename Pack<E, V>::type pack_load(const E* p) { return *(const typename Pack<E, V>::loose*)p; }
template <class E, int V> __device__ __forceinline__ void pack_store(E* p, typename Pack<E, V>::type v) { *(typename Pack<E, V>::loose*)p = v; }

// Draws of elements from number e on: the state of the draw that serves e, and e's place in it.
struct DropPlace {
    uint64_t state;
    uint32_t phase;
    __device__ __forceinline__ DropPlace(const DropRule& d, uint64_t e) : state(d.base + (e >> 2) * SPLITMIX_GAMMA), phase((uint32_t)e & 3) {}
    __device__ __forceinline__ DropPlace(uint64_t state, uint32_t phase) : state(state), phase(phase) {}
};

// The elements of a pack that are dropped become 0.  V a multiple of 4: a draw serves four of them; where the first one's number is no
// multiple of 4 (ALIGNED false) they straddle one draw more.  A field of 16 bits is kept if it is above T - 1 (threshold 1..65536).  In bf16
// the fields stand as the elements do: two of them in three packed instructions, the field less T - 1, at 0 and at 1 cut off, times the
// element's bits.  In fp32 16-bit comparisons for the lower halves of a draw's words, for the upper ones the word against (T - 1) 2^16 + 65535,
// so that no field is moved.
template <class E, int V, bool ALIGNED> __device__ __forceinline__ void drop_pack(const DropRule& d, DropPlace at, typename Pack<E, V>::type& v) {
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    const uint16_t low = (uint16_t)(d.threshold - 1);
    const uint32_t high = ((d.threshold - 1) << 16) | 0xFFFF;
    uint64_t word = splitmix64_mix(at.state);
    const bool halves = at.phase & 2;
    const uint32_t quarter = 16 * (at.phase & 1);
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        uint32_t lo = (uint32_t)word, hi = (uint32_t)(word >> 32);
        if (!ALIGNED || i + 4 < V) {
            at.state += SPLITMIX_GAMMA;
            word = splitmix64_mix(at.state);
        }
        if (!ALIGNED) {
            // In 32-bit steps.  (A 64-bit shift whose amount lies in the last of a wavefront's vector registers, at the end of eight, reads
            // another wavefront's instead: seen here as masks of a draw that were wrong now and then, in a kernel of 88 registers that
            // kept the amount in the 88th.  No kernel of the layers shifts 64 bits by an amount in a vector register.)
            uint32_t upper = (uint32_t)(word >> 32);
            asm("" : "+v"(upper), "+v"(hi));
            const uint32_t next = (uint32_t)word, mid = halves ? next : hi, last = halves ? upper : next;
            lo = halves ? hi : lo;
            lo = __builtin_amdgcn_alignbit(mid, lo, quarter);
            hi = __builtin_amdgcn_alignbit(last, mid, quarter);
        }
        if constexpr (sizeof(E) == 2) {
            typedef uint32_t words __attribute__((ext_vector_type(V / 2)));
            words w = __builtin_bit_cast(words, v);
            const uint32_t from = low * 0x10001u, fields[2] = {lo, hi};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t keep;                       // (as instructions: the compiler makes them comparisons and choices, twice as many)
                asm("v_pk_sub_u16 %0, %1, %2 clamp" : "=v"(keep) : "v"(fields[j]), "s"(from));
                asm("v_pk_min_u16 %0, %1, %2" : "=v"(keep) : "v"(keep), "s"(0x10001));
                w[i / 2 + j] = __builtin_bit_cast(uint32_t, (pair)(__builtin_bit_cast(pair, (uint32_t)w[i / 2 + j]) * __builtin_bit_cast(pair, keep)));
            }
            v = __builtin_bit_cast(typename Pack<E, V>::type, w);
        } else {
            v[i] = (uint16_t)lo > low ? v[i] : (E)0.f;
            v[i + 1] = lo > high ? v[i + 1] : (E)0.f;
            v[i + 2] = (uint16_t)hi > low ? v[i + 2] : (E)0.f;
            v[i + 3] = hi > high ? v[i + 3] : (E)0.f;
        }
    }
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__bf16 v) { return (float)v; }
template <class E> __device__ __forceinline__ E from_float(float v) { return (E)v; }     // bf16: nearest, ties to even

// Activation and slope.  SiLU: of t = -z log2 e (SILU_SCALE z; what multiplies z takes that factor), with the hardware's exponential and
// reciprocal: s = 1 / (1 + 2^t) = sigmoid(z) within a few 2^-24, and |z| 2^-24 more for the rounding of t.  z s and the slope
// s (1 + z (1 - s)) follow with z = t SILU_BACK.  ReLU: with the floor below which it cuts; none is a floor that nothing is below (forward:
// -inf, which leaves NaN and -inf what they are; backward: NaN, which compares as false).
constexpr float SILU_SCALE = -1.44269504088896341f, SILU_BACK = -0.69314718055994531f;
__device__ __forceinline__ float sigmoid_of(float t) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t)); }
// SiLU: without the factor SILU_BACK
template <bool SILU> __device__ __forceinline__ float activate(float z, float floor) {
    return SILU ? z * sigmoid_of(z) : __builtin_elementwise_maximum(z, floor);
}
template <bool SILU> __device__ __forceinline__ float through_slope(float g, float z, float floor) {
    if (SILU) {
        const float s = sigmoid_of(z), rest = __builtin_fmaf(-SILU_BACK, s, SILU_BACK);
        return g * (s * __builtin_fmaf(z, rest, 1.f));
    }
    return z <= floor ? 0.f : g;
}
#endif

}  // namespace kavg
