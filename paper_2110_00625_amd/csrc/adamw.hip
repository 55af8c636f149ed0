// AdamW over many tensors: one pass over parameter, gradient and both moments of every element (formulas: kavg.h).  34 vector instructions
// per element, 63 with states in 8 bits, beside 28 and 16 bytes: bound by memory.  A workgroup takes a piece of a row, a wavefront 256 values of it at a
// time, four per lane, which are the values that share the scales of an 8-bit state, so that a block's largest magnitude is six moves between lanes.  The
// tensors of a launch come as kernel arguments (a table in memory would have to be copied there by every call, or kept).
// 75M parameters in six tensors with a bf16 copy: 32 bits 360 us (6.3 TB/s; 412, 5.5 TB/s, where the states of three nets are stepped in turn and none of it
// is in the cache), 8 bits and gradients in bf16 190 (210).  13 small tensors 3.6 of a call of 10, which is the host's.  Steps on the way: streaming
// accesses past the cache 427 -> 366 (one tensor); codes and draws of 108 instructions per element, which were as long as the bytes, 240 -> 184.
#include "adamw.h"
#include "layers.h"
#include "split.h"
#include "wave_sum.h"
#include <algorithm>
#include <cmath>

namespace kavg {

namespace {

constexpr int T = 256, BLOCK = 256;
// Blocks that a wavefront has under way: 75M parameters with 1 / 2 / 4 of them 420 / 420 / 412 us, with states in 8 bits 210 / 217 / 221.  In the cache more
// wavefronts do better: 13 small tensors 3.6 for 4.9 us with 1 for 4 of them, 8M parameters 53 for 54.
constexpr int turns_of(int bits, bool stream) { return bits == 32 && stream ? 4 : 1; }
constexpr int piece_of(int bits, bool stream) { return T * 4 * turns_of(bits, stream); }
constexpr double CACHE = 256e6;                  // bytes behind the L2: tensors of more are gone by the next step
constexpr int MOST_TENSORS = 32;                 // of a launch: its arguments stay below four kilobytes

struct Table {
    uint32_t first[MOST_TENSORS + 1];            // pieces before each tensor, and in all
    int count;
    AdamwTensor tensor[MOST_TENSORS];
};
static_assert(sizeof(Table) + sizeof(AdamwRule) <= 4096, "kernel arguments");

// 1 - beta^t, in 64 bits (in 32, 1 - 0.999 would be off by a ten thousandth of itself)
__host__ __device__ inline double rest_of_power(double beta, uint64_t t) {
    double p = 1.;
    for (double b = beta; t; t >>= 1, b *= b) if (t & 1) p *= b;
    return 1. - p;
}

__host__ __device__ inline void at_step(AdamwRule& r, uint64_t t) {
    r.rate = (float)(r.lr / rest_of_power(r.exact1, t));
    r.root_scale = (float)(1. / sqrt(rest_of_power(r.exact2, t)));
}

struct Four { float v[4]; };

// four values of which n are there; STREAM: of tensors that no cache holds until the next step
template <bool STREAM, class E> __device__ __forceinline__ Four load_four(const E* p, int n) {
    Four f;
    if (n >= 4) {
        const auto at = (const typename Pack<E, 4>::loose*)p;
        const typename Pack<E, 4>::type v = STREAM ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
        for (int k = 0; k < 4; ++k) f.v[k] = to_float(v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) f.v[k] = k < n ? to_float(p[k]) : 0.f;
    }
    return f;
}
template <bool STREAM> __device__ __forceinline__ void store_four(float* p, const Four& f, int n) {
    if (n >= 4) {
        const Pack<float, 4>::type v = {f.v[0], f.v[1], f.v[2], f.v[3]};
        const auto at = (Pack<float, 4>::loose*)p;
        if (STREAM) __builtin_nontemporal_store(v, at);
        else *at = v;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) if (k < n) p[k] = f.v[k];
    }
}
typedef uint32_t loose_word __attribute__((aligned(1)));
template <bool STREAM> __device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n) {
    const auto at = (const loose_word*)p;
    if (n >= 4) return STREAM ? __builtin_nontemporal_load(at) : *at;
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) w |= (uint32_t)p[k] << (8 * k);
    return w;
}
template <bool STREAM> __device__ __forceinline__ void store_codes(uint8_t* p, uint32_t w, int n) {
    const auto at = (loose_word*)p;
    if (n >= 4) {
        if (STREAM) __builtin_nontemporal_store(w, at);
        else *at = w;
        return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) p[k] = (uint8_t)(w >> (8 * k));
}
// four e4m3 codes times their scale (exact: a power of two)
__device__ __forceinline__ Four decoded(uint32_t w, float scale) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return {{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale}};
}

// Exponent field of the scale of a block whose largest finite magnitude has these bits: 2^(k-8) for 2^(k-1) c <= magnitude < 2^k c.  (c lies
// below 448/256 and where no beta-weighted sum of an e4m3 and a bf16 value falls, so that no scale depends on the order of roundings.)
constexpr uint32_t BORDER = 0x5DB3D7;
__device__ __forceinline__ uint32_t scale_field(uint32_t most) {
    const int f = (int)((most + 0x800000u - BORDER) >> 23) - 8;
    return (uint32_t)(f < 1 ? 1 : f);
}
__device__ __forceinline__ float power(uint32_t field) { return __builtin_bit_cast(float, field << 23); }
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < INFINITY; }

// bits of the largest of non-negative values over the wavefront, in all 64 lanes' scalar: NaN above infinity above the others
template <int CTRL> __device__ __forceinline__ uint32_t max_of_move(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true)); }
__device__ __forceinline__ uint32_t largest(const Four& f) {
    uint32_t x = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) x = max(x, __builtin_bit_cast(uint32_t, f.v[k]) & 0x7FFFFFFFu);
    x = max_of_move<0xB1>(x);          // quad_perm [1,0,3,2]
    x = max_of_move<0x4E>(x);          // quad_perm [2,3,0,1]
    x = max_of_move<0x141>(x);         // row_half_mirror
    x = max_of_move<0x140>(x);         // row_mirror
    x = max_of_move<0x142>(x);         // row_bcast:15, each row's last lane to the next row
    x = max_of_move<0x143>(x);         // row_bcast:31
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
constexpr uint32_t INFINITE = 0x7F800000;
// ... of those that are finite
__device__ __forceinline__ uint32_t largest_finite(Four f) {
#pragma unroll
    for (int k = 0; k < 4; ++k) f.v[k] = finite(f.v[k]) ? f.v[k] : 0.f;
    return largest(f);
}

constexpr uint32_t CODE_NAN = 0x7F;

// to nearest, by the hardware's conversion
__device__ __forceinline__ uint32_t coded_nearest(const Four& f, float inverse) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(f.v[0] * inverse, f.v[1] * inverse, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f.v[2] * inverse, f.v[3] * inverse, w, true);
}

// Down or up by a draw: with u the distance of e4m3's values around q, floor(q / u), one more where remainder + draw reaches one.  The codes
// count those distances: eight to an octave, from 2^-6 on; below it they are what they are there.
__device__ __forceinline__ uint32_t coded_drawn(float q, uint32_t field16) {
    const int e = max(__builtin_amdgcn_frexp_expf(q), -5);
    const float steps = __builtin_ldexpf(q, 4 - e), down = __builtin_floorf(steps);
    const float draw = (float)(2 * field16 + 1) * 0x1p-17f;
    const int code = (int)down + ((steps - down) + draw >= 1.f ? 1 : 0) + 8 * (e + 5);
    return (uint32_t)(q > 0.f ? max(code, 1) : 0);
}
// The same of four values from 2^-6 on: there the code is the value's bits from the third of its mantissa on, and the draw, as wide as the others and a half
// of their last place more, is added to those.  (Moved up by four places: a code is the top byte.)
__device__ __forceinline__ uint32_t coded_drawn_normal(const Four& q, uint32_t lo16, uint32_t hi16) {
    constexpr uint32_t REST = (8u << 4) - (960u << 24);
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t w = k < 2 ? lo16 : hi16, field = (k & 1 ? w >> 8 : w << 8) & 0xFFFF00u;
        u[k] = (__builtin_bit_cast(uint32_t, q.v[k]) << 4) + (field + REST);
    }
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0703), hi = __builtin_amdgcn_perm(u[3], u[2], 0x07030C0C);
    return lo | hi;
}

// the 16-bit fields of elements e .. e+3 (two to a word): of the draw with this state, or from the (e mod 4)-th field on into the next
__device__ __forceinline__ void draw_four(uint64_t state, uint32_t phase, uint32_t* lo, uint32_t* hi) {
    const uint64_t word = splitmix64_mix(state);
    *lo = (uint32_t)word;
    *hi = (uint32_t)(word >> 32);
    if (phase) {
        const uint64_t more = splitmix64_mix(state + SPLITMIX_GAMMA);
        const uint32_t next = (uint32_t)more, last0 = (uint32_t)(more >> 32), quarter = 16 * (phase & 1);
        const bool halves = phase & 2;
        const uint32_t a = halves ? *hi : *lo, b = halves ? next : *hi, c = halves ? last0 : next;
        *lo = __builtin_amdgcn_alignbit(b, a, quarter);       // (32-bit steps: see layers.h)
        *hi = __builtin_amdgcn_alignbit(c, b, quarter);
    }
}

// New moments (every operation rounded by itself, as the interface says, so that 8-bit states are a matter of bits).
__device__ __forceinline__ void moments(const AdamwRule& r, float g, float& m, float& v, float& root) {
#pragma clang fp contract(off)
    m = m * r.beta1 + g * r.rest1;
    v = v * r.beta2 + (g * g) * r.rest2;
    root = __builtin_sqrtf(v);
}
// The parameter, with the hardware's reciprocal (one unit in the last place of the change), which takes and gives no subnormal numbers.  The denominator is
// normal, zero or infinite where eps is: a root of fp32 is normal or zero, and its factor is 1 at least; where eps lies outside of what has a normal
// reciprocal the quotient is taken in 64 bits.
template <bool WIDE> __device__ __forceinline__ float stepped(const AdamwRule& r, float p, float decay, float m, float root) {
    if (WIDE) return (float)((double)p * decay - r.rate * (m / ((double)root * r.root_scale + r.exact_eps)));
    const float change = m * __builtin_amdgcn_rcpf(__builtin_fmaf(root, r.root_scale, r.eps));
    return __builtin_fmaf(p, decay, -(r.rate * change));
}

// One wavefront's part of a piece: TURNS blocks of its row, the t-th from `first` + t T/64 BLOCK on.  WHOLE: all of them are there.
template <int BITS, class G, bool STREAM, bool WIDE, bool WHOLE>
__device__ __forceinline__ void step_piece(const AdamwTensor& t, const AdamwRule& rule, uint32_t row, int64_t first, int lane, uint64_t lane_draw) {
    const int64_t states = row * t.cols + first, blocks = (t.cols + BLOCK - 1) / BLOCK, left = t.cols - first;
    float* param = t.param + row * t.param_stride + first;
    const G* grad = (const G*)t.grad + row * t.grad_stride + first;
    const float decay = (float)(1. - rule.lr * t.decay);
    const uint64_t draw0 = rule.seed + (1 + ((uint64_t)t.site << 40) + ((uint64_t)states >> 2)) * SPLITMIX_GAMMA;      // of the first lane
    constexpr int APART = T / 64 * BLOCK, TURNS = turns_of(BITS, STREAM);
    Four p[TURNS], g[TURNS], m[TURNS], v[TURNS];
    uint32_t mc[TURNS], vc[TURNS];
    float ms[TURNS], vs[TURNS];
    int n[TURNS];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const uint32_t at = i * APART + lane * 4;
        n[i] = WHOLE ? 4 : (int)max((int64_t)0, min((int64_t)4, left - (int64_t)at));
        p[i] = load_four<STREAM>(param + at, n[i]);
        g[i] = load_four<STREAM>(grad + at, n[i]);
        if constexpr (BITS == 32) {
            m[i] = load_four<STREAM>((const float*)t.m + states + at, n[i]);
            v[i] = load_four<STREAM>((const float*)t.v + states + at, n[i]);
        } else {
            mc[i] = load_codes<STREAM>((const uint8_t*)t.m + states + at, n[i]);
            vc[i] = load_codes<STREAM>((const uint8_t*)t.v + states + at, n[i]);
            const int64_t block = row * blocks + min((first + i * APART) / BLOCK, blocks - 1);
            ms[i] = t.m_scale[block];
            vs[i] = t.v_scale[block];
        }
    }
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const uint32_t at = i * APART + lane * 4;
        if (!WHOLE && i * APART >= left) break;             // (a whole wavefront)
        if constexpr (BITS == 8) {
            m[i] = decoded(mc[i], ms[i]);
            v[i] = decoded(vc[i], vs[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i].v[k] *= v[i].v[k];
        }
        Four root;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            moments(rule, g[i].v[k] * rule.grad_scale, m[i].v[k], v[i].v[k], root.v[k]);
            p[i].v[k] = stepped<WIDE>(rule, p[i].v[k], decay, m[i].v[k], root.v[k]);
        }
        store_four<STREAM>(param + at, p[i], n[i]);
        if (t.copy) {
            uint16_t* copy = t.copy + row * t.copy_stride + first + at;
            Pack<uint16_t, 4>::type c;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float value = p[i].v[k];
                c[k] = (uint16_t)split_hi(__builtin_bit_cast(uint32_t, value));
            }
            if (n[i] >= 4) *(Pack<uint16_t, 4>::loose*)copy = c;
            else {
#pragma unroll
                for (int k = 0; k < 4; ++k) if (k < n[i]) copy[k] = c[k];
            }
        }
        if constexpr (BITS == 32) {
            store_four<STREAM>((float*)t.m + states + at, m[i], n[i]);
            store_four<STREAM>((float*)t.v + states + at, v[i], n[i]);
        } else {
            if (!WHOLE) {
#pragma unroll
                for (int k = 0; k < 4; ++k) if (k >= n[i]) m[i].v[k] = root.v[k] = 0.f;
            }
            uint32_t most_m = largest(m[i]), most_r = largest(root);
            const bool bad = most_m >= INFINITE || most_r >= INFINITE;
            if (bad) { most_m = largest_finite(m[i]); most_r = largest_finite(root); }
            const uint32_t fm = scale_field(most_m), fv = scale_field(most_r);
            uint32_t lo16, hi16, m_codes = coded_nearest(m[i], power(254 - fm)), v_codes = 0;
            draw_four(draw0 + i * (APART / 4) * SPLITMIX_GAMMA + lane_draw, (uint32_t)states & 3, &lo16, &hi16);
            Four q;
            float least = INFINITY;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                q.v[k] = root.v[k] * power(254 - fv);
                least = fminf(least, q.v[k]);
            }
            if (!bad && __builtin_amdgcn_ballot_w64(!(least >= 0x1p-6f)) == 0) v_codes = coded_drawn_normal(q, lo16, hi16);
            else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t word = k < 2 ? lo16 : hi16;
                    uint32_t code = coded_drawn(q.v[k], k & 1 ? word >> 16 : word & 0xFFFF);
                    if (!finite(root.v[k])) code = CODE_NAN;
                    if (!finite(m[i].v[k])) m_codes = (m_codes & ~(0xFFu << (8 * k))) | CODE_NAN << (8 * k);
                    v_codes |= code << (8 * k);
                }
            }
            store_codes<STREAM>((uint8_t*)t.m + states + at, m_codes, n[i]);
            store_codes<STREAM>((uint8_t*)t.v + states + at, v_codes, n[i]);
            if (lane == 0) {
                const int64_t block = row * blocks + (first + i * APART) / BLOCK;
                t.m_scale[block] = power(fm);
                t.v_scale[block] = power(fv);
            }
        }
    }
}

template <int BITS, class G, bool STREAM, bool WIDE>
__global__ void __launch_bounds__(T) adamw_kernel(Table table, AdamwRule rule) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (rule.lr_dev) rule.lr = *rule.lr_dev;
    if (rule.grad_scale_dev) rule.grad_scale = *rule.grad_scale_dev;
    if (rule.step_dev || rule.lr_dev) {
        // (the host's step went into the seed and the rate already)
        const int64_t t = rule.step_dev ? max(*rule.step_dev, (int64_t)1) : (int64_t)rule.step;
        if (rule.step_dev) rule.seed += (uint64_t)t;
        at_step(rule, (uint64_t)t);
    }
    const uint64_t lane_draw = (uint64_t)lane * SPLITMIX_GAMMA;
    const uint32_t total = table.first[table.count];
    for (uint32_t piece = blockIdx.x; piece < total; piece += gridDim.x) {
        int lo = 0, hi = table.count;                       // the last tensor that begins at or before it
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (table.first[mid] <= piece) lo = mid; else hi = mid;
        }
        const AdamwTensor& t = table.tensor[lo];
        const uint32_t in = piece - table.first[lo], row = in / t.pieces;
        const int64_t begin = (int64_t)(in - row * t.pieces) * piece_of(BITS, STREAM), first = begin + wave * BLOCK;
        if (begin + piece_of(BITS, STREAM) <= t.cols) step_piece<BITS, G, STREAM, WIDE, true>(t, rule, row, first, lane, lane_draw);
        else if (first < t.cols) step_piece<BITS, G, STREAM, WIDE, false>(t, rule, row, first, lane, lane_draw);
    }
}

template <int BITS, class G>
hipError_t start(const Table& table, const AdamwRule& rule, bool stream, hipStream_t st) {
    const dim3 grid(std::min<uint32_t>(table.first[table.count], 1u << 22));
    if (rule.wide) adamw_kernel<BITS, G, false, true><<<grid, dim3(T), 0, st>>>(table, rule);
    else if (stream) adamw_kernel<BITS, G, true, false><<<grid, dim3(T), 0, st>>>(table, rule);
    else adamw_kernel<BITS, G, false, false><<<grid, dim3(T), 0, st>>>(table, rule);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(int bits, int grad_dtype, const AdamwRule& given, const kavg_adamw_tensor* tensors, int count, hipStream_t st) {
    AdamwRule rule = given;
    if (!rule.step_dev) { at_step(rule, rule.step); rule.seed += rule.step; }
    double bytes = 0.;
    for (int i = 0; i < count; ++i) bytes += (double)tensors[i].rows * tensors[i].cols * (4 + (grad_dtype == KAVG_BF16 ? 2 : 4) + bits / 4);
    const bool stream = bytes > CACHE && !rule.wide;
    Table table;
    table.count = 0;
    table.first[0] = 0;
    hipError_t e = hipSuccess;
    auto flush = [&] {
        if (table.count && e == hipSuccess)
            e = bits == 32 ? (grad_dtype == KAVG_BF16 ? start<32, __bf16>(table, rule, stream, st) : start<32, float>(table, rule, stream, st))
                           : (grad_dtype == KAVG_BF16 ? start<8, __bf16>(table, rule, stream, st) : start<8, float>(table, rule, stream, st));
        table.count = 0;
    };
    for (int i = 0; i < count; ++i) {
        const kavg_adamw_tensor& t = tensors[i];
        if (!t.rows || !t.cols) continue;
        AdamwTensor a = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.cols, t.param_stride, t.grad_stride, t.copy_stride, (uint32_t)t.rows, 0, t.weight_decay, (uint32_t)i};
        // rows without gaps are one row (blocks of 256 stay what they are where they fill the rows)
        if (t.param_stride == t.cols && t.grad_stride == t.cols && (!t.copy || t.copy_stride == t.cols) && (bits == 32 || t.cols % BLOCK == 0)) {
            a.cols *= t.rows;
            a.rows = 1;
        }
        a.pieces = (uint32_t)((a.cols + piece_of(bits, stream) - 1) / piece_of(bits, stream));
        const uint64_t more = (uint64_t)a.rows * a.pieces;              // below 2^32, from the limits of the call
        if (table.count == MOST_TENSORS || table.first[table.count] + more >= (uint64_t)1 << 31) flush();
        table.tensor[table.count] = a;
        table.first[table.count + 1] = table.first[table.count] + (uint32_t)more;
        ++table.count;
    }
    flush();
    return e;
}

}  // namespace kavg
