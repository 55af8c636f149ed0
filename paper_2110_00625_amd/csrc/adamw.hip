// AdamW over many tensors: one pass over parameter, gradient and both moments of every element (formulas: kavg.h).  Some forty vector
// instructions per element, 120 with states in 8 bits, beside 28 and 16 bytes: bound by memory.  A workgroup takes a piece of a row, a wavefront
// 256 values of it at a time, four per lane, which are the values that share the scales of an 8-bit state, so that a block's largest
// magnitude is a butterfly over the lanes.  The tensors of a launch come as kernel arguments (a table in memory would have to
// be copied there by every call, or kept).
#include "adamw.h"
#include "layers.h"
#include "split.h"
#include "wave_sum.h"
#include <algorithm>
#include <cmath>

namespace kavg {

namespace {

constexpr int T = 256, BLOCK = 256, TURNS = 2, PIECE = T * 4 * TURNS;
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

template <class E> __device__ __forceinline__ Four load_four(const E* p, int n) {
    Four f;
    if (n >= 4) {
        const auto v = pack_load<E, 4>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) f.v[k] = to_float(v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) f.v[k] = k < n ? to_float(p[k]) : 0.f;
    }
    return f;
}
__device__ __forceinline__ void store_four(float* p, const Four& f, int n) {
    if (n >= 4) {
        Pack<float, 4>::type v = {f.v[0], f.v[1], f.v[2], f.v[3]};
        pack_store<float, 4>(p, v);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) if (k < n) p[k] = f.v[k];
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int n) {
    typedef uint32_t loose __attribute__((aligned(1)));
    if (n >= 4) return *(const loose*)p;
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < n) w |= (uint32_t)p[k] << (8 * k);
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, uint32_t w, int n) {
    typedef uint32_t loose __attribute__((aligned(1)));
    if (n >= 4) { *(loose*)p = w; return; }
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

__device__ __forceinline__ uint32_t largest(const Four& f) {
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) most = fmaxf(most, finite(f.v[k]) ? __builtin_fabsf(f.v[k]) : 0.f);
    most = butterfly(most, [](float a, float b) { return fmaxf(a, b); });
    return __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, most));
}

constexpr uint32_t CODE_NAN = 0x7F;

// to nearest, by the hardware's conversion
__device__ __forceinline__ uint32_t coded_nearest(const Four& f, float inverse) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f.v[0] * inverse, f.v[1] * inverse, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f.v[2] * inverse, f.v[3] * inverse, w, true);
#pragma unroll
    for (int k = 0; k < 4; ++k) if (!finite(f.v[k])) w = (w & ~(0xFF << (8 * k))) | (int)(CODE_NAN << (8 * k));
    return (uint32_t)w;
}

// Down or up by a draw: with u the distance of e4m3's values around q, floor(q / u), one more where remainder + draw reaches one.  The codes
// count those distances: eight to an octave, from 2^-6 on; below it they are what they are there.
__device__ __forceinline__ uint32_t coded_drawn(float r, float inverse, uint32_t field16) {
    if (!finite(r)) return CODE_NAN;
    const float q = r * inverse;
    const int e = max(__builtin_amdgcn_frexp_expf(q), -5);
    const float steps = __builtin_ldexpf(q, 4 - e), down = __builtin_floorf(steps);
    const float draw = (float)(2 * field16 + 1) * 0x1p-17f;
    const int code = (int)down + ((steps - down) + draw >= 1.f ? 1 : 0) + 8 * (e + 5);
    return (uint32_t)(q > 0.f ? max(code, 1) : 0);
}

// the 16-bit fields of elements e .. e+3 (two to a word), whose draws have states base + (e/4) gamma and, unless aligned, the next
__device__ __forceinline__ void draw_four(uint64_t base, uint64_t e, bool aligned, uint32_t* lo, uint32_t* hi) {
    const uint64_t state = base + (e >> 2) * SPLITMIX_GAMMA, word = splitmix64_mix(state);
    *lo = (uint32_t)word;
    *hi = (uint32_t)(word >> 32);
    if (!aligned) {
        const uint64_t more = splitmix64_mix(state + SPLITMIX_GAMMA);
        const uint32_t next = (uint32_t)more, last0 = (uint32_t)(more >> 32), quarter = 16 * ((uint32_t)e & 1);
        const bool halves = e & 2;
        const uint32_t a = halves ? *hi : *lo, b = halves ? next : *hi, c = halves ? last0 : next;
        *lo = __builtin_amdgcn_alignbit(b, a, quarter);       // (32-bit steps: see layers.h)
        *hi = __builtin_amdgcn_alignbit(c, b, quarter);
    }
}

// new moments (every operation rounded by itself, as the interface says, so that 8-bit states are a matter of bits) and parameter
__device__ __forceinline__ void update(const AdamwRule& r, float g, float decay, float& p, float& m, float& v, float& root) {
#pragma clang fp contract(off)
    m = m * r.beta1 + g * r.rest1;
    v = v * r.beta2 + (g * g) * r.rest2;
    root = __builtin_sqrtf(v);
    p = p * decay - r.rate * (m / (root * r.root_scale + r.eps));
}

template <int BITS, class G>
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
    const uint32_t total = table.first[table.count];
    for (uint32_t piece = blockIdx.x; piece < total; piece += gridDim.x) {
        int lo = 0, hi = table.count;                       // the last tensor that begins at or before it
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (table.first[mid] <= piece) lo = mid; else hi = mid;
        }
        const AdamwTensor& t = table.tensor[lo];
        const uint32_t in = piece - table.first[lo], row = in / t.pieces;
        const int64_t col0 = (int64_t)(in - row * t.pieces) * PIECE;
        float* param = t.param + row * t.param_stride;
        const G* grad = (const G*)t.grad + row * t.grad_stride;
        const int64_t states = row * t.cols;
        const float decay = (float)(1. - rule.lr * t.decay);
        const int64_t blocks = (t.cols + BLOCK - 1) / BLOCK;
        const bool aligned = t.cols % 4 == 0;
        const uint64_t base = rule.seed + (1 + ((uint64_t)t.site << 40)) * SPLITMIX_GAMMA;

        Four p[TURNS], g[TURNS], m[TURNS], v[TURNS];
        uint32_t mc[TURNS], vc[TURNS];
        float ms[TURNS], vs[TURNS];
        int n[TURNS];
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int64_t block = col0 + (i * (T / 64) + wave) * BLOCK, col = block + lane * 4;
            n[i] = (int)max((int64_t)0, min((int64_t)4, t.cols - col));
            p[i] = load_four(param + col, n[i]);
            g[i] = load_four(grad + col, n[i]);
            if constexpr (BITS == 32) {
                m[i] = load_four((const float*)t.m + states + col, n[i]);
                v[i] = load_four((const float*)t.v + states + col, n[i]);
            } else {
                mc[i] = load_codes((const uint8_t*)t.m + states + col, n[i]);
                vc[i] = load_codes((const uint8_t*)t.v + states + col, n[i]);
                const int64_t at = row * blocks + min(block / BLOCK, blocks - 1);
                ms[i] = t.m_scale[at];
                vs[i] = t.v_scale[at];
            }
        }
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            const int64_t block = col0 + (i * (T / 64) + wave) * BLOCK, col = block + lane * 4;
            if (block >= t.cols) break;                     // (a whole wavefront)
            if constexpr (BITS == 8) {
                m[i] = decoded(mc[i], ms[i]);
                v[i] = decoded(vc[i], vs[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i].v[k] *= v[i].v[k];
            }
            Four root;
#pragma unroll
            for (int k = 0; k < 4; ++k) update(rule, g[i].v[k] * rule.grad_scale, decay, p[i].v[k], m[i].v[k], v[i].v[k], root.v[k]);
            store_four(param + col, p[i], n[i]);
            if (t.copy) {
                uint16_t* copy = t.copy + row * t.copy_stride + col;
                typedef uint16_t four __attribute__((ext_vector_type(4)));
                typedef four loose __attribute__((aligned(2)));
                four c;
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] = (uint16_t)split_hi(__builtin_bit_cast(uint32_t, p[i].v[k]));
                if (n[i] >= 4) *(loose*)copy = c;
                else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) if (k < n[i]) copy[k] = c[k];
                }
            }
            if constexpr (BITS == 32) {
                store_four((float*)t.m + states + col, m[i], n[i]);
                store_four((float*)t.v + states + col, v[i], n[i]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) if (k >= n[i]) m[i].v[k] = root.v[k] = 0.f;
                const uint32_t fm = scale_field(largest(m[i])), fv = scale_field(largest(root));
                uint32_t lo16, hi16, codes = 0;
                draw_four(base, (uint64_t)(states + col), aligned, &lo16, &hi16);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t word = k < 2 ? lo16 : hi16;
                    codes |= coded_drawn(root.v[k], power(254 - fv), k & 1 ? word >> 16 : word & 0xFFFF) << (8 * k);
                }
                store_codes((uint8_t*)t.m + states + col, coded_nearest(m[i], power(254 - fm)), n[i]);
                store_codes((uint8_t*)t.v + states + col, codes, n[i]);
                if (lane == 0) {
                    const int64_t at = row * blocks + block / BLOCK;
                    t.m_scale[at] = power(fm);
                    t.v_scale[at] = power(fv);
                }
            }
        }
    }
}

template <int BITS, class G>
hipError_t start(const Table& table, const AdamwRule& rule, hipStream_t st) {
    const uint32_t total = table.first[table.count];
    adamw_kernel<BITS, G><<<dim3(std::min<uint32_t>(total, 1u << 22)), dim3(T), 0, st>>>(table, rule);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(int bits, int grad_dtype, const AdamwRule& given, const kavg_adamw_tensor* tensors, int count, hipStream_t st) {
    AdamwRule rule = given;
    if (!rule.step_dev) { at_step(rule, rule.step); rule.seed += rule.step; }
    Table table;
    table.count = 0;
    table.first[0] = 0;
    hipError_t e = hipSuccess;
    auto flush = [&] {
        if (table.count && e == hipSuccess)
            e = bits == 32 ? (grad_dtype == KAVG_BF16 ? start<32, __bf16>(table, rule, st) : start<32, float>(table, rule, st))
                           : (grad_dtype == KAVG_BF16 ? start<8, __bf16>(table, rule, st) : start<8, float>(table, rule, st));
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
        a.pieces = (uint32_t)((a.cols + PIECE - 1) / PIECE);
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
