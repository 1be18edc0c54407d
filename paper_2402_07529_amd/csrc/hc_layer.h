// hc_layer.h -- device-side pieces of the layer operators (include/hc_train.h):
// the generator of dropout's masks, activations and their slopes, and rows read
// and written eight elements at a time.
#pragma once

#include "hc_device.h"
#include "hc_train_internal.h"

namespace hc {

// ---- dropout's masks -------------------------------------------------------------

// One call's masks: the eight elements 8 c .. 8 c + 7 of row r share a call of
// Philox4x32-10 (Salmon et al. 2011) with key = seed and counter = (c, r, draw),
// 16 bits an element, so that a mask depends on an element's place alone and is
// made again where it is needed.  16 bits rather than 32 because the generator
// bounds the pass otherwise: a call is 20 products of 32 bits, which run at a
// quarter of the rate.
struct Masks {
    uint32_t k0, k1, c2, c3;
    uint32_t limit;  // dropped where the 16 bits are below it
    float scale;     // of what is kept
};

__device__ __forceinline__ Masks masks_of(const Dropout& d) {
    const uint64_t draw = d.draw + (d.counter ? *d.counter : 0);
    return {(uint32_t)d.seed, (uint32_t)(d.seed >> 32), (uint32_t)draw, (uint32_t)(draw >> 32),
            d.limit, d.scale};
}

struct MaskBits {
    uint32_t w[4];
    __device__ __forceinline__ bool kept(int e, uint32_t limit) const {
        return ((e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) >= limit;
    }
};

__device__ __forceinline__ MaskBits mask_bits(const Masks& m, uint32_t row, uint32_t group) {
    uint32_t a = group, b = row, c = m.c2, d = m.c3, k0 = m.k0, k1 = m.k1;
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
        a = __builtin_amdgcn_bitop3_b32((uint32_t)(q >> 32), b, k0, 0x96);  // exclusive or
        b = (uint32_t)q;
        c = __builtin_amdgcn_bitop3_b32((uint32_t)(p >> 32), d, k1, 0x96);
        d = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{a, b, c, d}};
}

// v times its mask: a dropped element is 0 whatever it was.
__device__ __forceinline__ void drop8(const Masks& m, uint32_t row, uint32_t group, float (&v)[8]) {
    const MaskBits bits = mask_bits(m, row, group);
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = bits.kept(e, m.limit) ? v[e] * m.scale : 0.0f;
}

// ---- activations -----------------------------------------------------------------

// exp of the type's accuracy.  The hardware's 2^p is within a unit of 24 bits, but
// p = v log2 e is rounded, which is |v| such units of the result: far below half a
// unit of 11 bits, and for fp32 put right by the first term of what was lost.
template <typename T> __device__ __forceinline__ float exp_of(float v) {
    constexpr float kLog2e = 1.44269504088896341f, kLog2eRest = 1.92596299e-8f;
    if constexpr (sizeof(T) != 4) return __builtin_amdgcn_exp2f(v * kLog2e);
    v = v > 88.0f ? 88.0f : v < -104.0f ? -104.0f : v;  // infinity would meet its correction
    const float p = v * kLog2e, rest = __builtin_fmaf(v, kLog2e, -p) + v * kLog2eRest;
    const float e = __builtin_amdgcn_exp2f(p);
    return __builtin_fmaf(e, 0.69314718055994531f * rest, e);
}

// v from below at a finite value, where the functions are 0 already in fp32: what
// is left of minus infinity then is the limit, not infinity times zero.  NaN stays.
__device__ __forceinline__ float above(float v, float least) { return v < least ? least : v; }

// The normal distribution's Phi(z) and density phi(z): Phi(-a) = exp(-a^2 / 2) G(a),
// G by a polynomial of eighth degree in 1 / (1 + 0.24 a) fitted to it in relative
// error (4.3e-7, 7.3e-7 with fp32 arithmetic); 21 operations, where the device
// library's erfc and exp take some 60 and make the tiles' results too long to unroll.
template <typename T> __device__ __forceinline__ void normal(float z, float& cdf, float& density) {
    const float a = fabsf(z), e = exp_of<T>(-0.5f * z * z);
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.24f * a);
    float g = -0.052992403507232666f;
    g = g * t + 0.15279580652713776f;
    g = g * t - 0.06570429354906082f;
    g = g * t + 0.11838865280151367f;
    g = g * t + 0.06339804083108902f;
    g = g * t + 0.09283839911222458f;
    g = g * t + 0.0955221951007843f;
    g = g * t + 0.09575378894805908f;
    g *= t * e;
    cdf = z < 0.0f ? g : 1.0f - g;
    density = 0.39894228040143268f * e;
}

// 1 / v within a unit of 24 bits.
__device__ __forceinline__ float inverse_of(float v) { return __builtin_amdgcn_rcpf(v); }

template <typename T> __device__ __forceinline__ float logistic(float z) {
    return inverse_of(1.0f + exp_of<T>(-z));
}

// The logistic function's slope e / (1 + e)^2, e = exp(-|z|): nothing cancels.
template <typename T> __device__ __forceinline__ float logistic_slope(float z) {
    const float e = exp_of<T>(-fabsf(z)), r = inverse_of(1.0f + e);
    return e * r * r;
}

// Near 0, where the quotient would cancel, the series up to z^11, 4e-9 off.
template <typename T> __device__ __forceinline__ float hyperbolic(float z) {
    const float s = z * z, e = exp_of<T>(-2.0f * fabsf(z));
    const float q = (1.0f - e) * inverse_of(1.0f + e);
    float c = -8.8632355299e-3f;
    c = c * s + 2.1869488536e-2f;
    c = c * s - 5.3968253968e-2f;
    c = c * s + 1.3333333333e-1f;
    c = c * s - 3.3333333333e-1f;
    return s < 0.1f ? z + z * s * c : __builtin_copysignf(q, z);
}

template <typename T> __device__ __forceinline__ float activate(uint32_t act, float z) {
    switch (act) {
        case HC_ACT_RELU: return z < 0.0f ? 0.0f : z;
        case HC_ACT_GELU: {
            float cdf, density;
            const float v = above(z, -64.0f);
            normal<T>(v, cdf, density);
            return v * cdf;
        }
        case HC_ACT_SILU: {
            const float v = above(z, -128.0f);
            return v * logistic<T>(v);
        }
        case HC_ACT_TANH: return hyperbolic<T>(z);
        case HC_ACT_SIGMOID: return logistic<T>(z);
        default: return z;
    }
}

// The activation's slope at z, times g.
template <typename T> __device__ __forceinline__ float backward(uint32_t act, float z, float g) {
    switch (act) {
        case HC_ACT_RELU: return z > 0.0f ? g : z != z ? z : 0.0f;
        case HC_ACT_GELU: {
            float cdf, density;
            float v = above(z, -64.0f);
            v = v > 64.0f ? 64.0f : v;
            normal<T>(v, cdf, density);
            return g * (cdf + v * density);
        }
        case HC_ACT_SILU: {
            float v = above(z, -128.0f);
            v = v > 128.0f ? 128.0f : v;
            return g * (logistic<T>(v) + v * logistic_slope<T>(v));
        }
        case HC_ACT_TANH: return g * (4.0f * logistic_slope<T>(2.0f * z));
        case HC_ACT_SIGMOID: return g * logistic_slope<T>(z);
        default: return g;
    }
}

// Eight at once: one branch on the activation.
template <typename T> __device__ __forceinline__ void activate8(uint32_t act, float (&v)[8]) {
    switch (act) {
#define HC_CASE(ACT)                                          \
    case ACT:                                                 \
        _Pragma("unroll") for (int e = 0; e < 8; e++) v[e] = activate<T>(ACT, v[e]); \
        break;
        HC_CASE(HC_ACT_RELU) HC_CASE(HC_ACT_GELU) HC_CASE(HC_ACT_SILU) HC_CASE(HC_ACT_TANH) HC_CASE(HC_ACT_SIGMOID)
#undef HC_CASE
        default: break;
    }
}

template <typename T> __device__ __forceinline__ void backward8(uint32_t act, const float (&z)[8], float (&v)[8]) {
    switch (act) {
#define HC_CASE(ACT)                                          \
    case ACT:                                                 \
        _Pragma("unroll") for (int e = 0; e < 8; e++) v[e] = backward<T>(ACT, z[e], v[e]); \
        break;
        HC_CASE(HC_ACT_RELU) HC_CASE(HC_ACT_GELU) HC_CASE(HC_ACT_SILU) HC_CASE(HC_ACT_TANH) HC_CASE(HC_ACT_SIGMOID)
#undef HC_CASE
        default: break;
    }
}

// ---- eight elements of a row -----------------------------------------------------

template <typename T> struct Eight {
    typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

// count: how many of them there are; the others are 0 and not read.
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ p, uint32_t count, float (&v)[8]) {
    if (count >= 8) {
        const typename Eight<T>::V t = *reinterpret_cast<const typename Eight<T>::V*>(p);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (float)t[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (uint32_t)e < count ? (float)p[e] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void load8_raw(const T* __restrict__ p, uint32_t count, T (&v)[8]) {
    if (count >= 8) {
        const typename Eight<T>::V t = *reinterpret_cast<const typename Eight<T>::V*>(p);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = t[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (uint32_t)e < count ? p[e] : (T)0.0f;
    }
}

template <typename T> __device__ __forceinline__ void store8(T* p, uint32_t count, const float (&v)[8]) {
    if (count >= 8) {
        typename Eight<T>::V t;
#pragma unroll
        for (int e = 0; e < 8; e++) t[e] = (T)v[e];
        *reinterpret_cast<typename Eight<T>::V*>(p) = t;
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if ((uint32_t)e < count) p[e] = (T)v[e];
    }
}

// The same past the caches, for what is read or written once.
template <typename T>
__device__ __forceinline__ void load8_past(const T* __restrict__ p, uint32_t count, float (&v)[8]) {
    if (count >= 8) {
        typedef typename Eight<T>::V V;
        const V t = __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (float)t[e];
    } else {
        load8(p, count, v);
    }
}

template <typename T> __device__ __forceinline__ void store8_past(T* p, uint32_t count, const float (&v)[8]) {
    if (count >= 8) {
        typename Eight<T>::V t;
#pragma unroll
        for (int e = 0; e < 8; e++) t[e] = (T)v[e];
        __builtin_nontemporal_store(t, reinterpret_cast<typename Eight<T>::V*>(p));
    } else {
        store8(p, count, v);
    }
}

// Fixed point: the nearest whole number, ties to even, saturating at +-(2^31 - 1)
// (NaN: 0).
__device__ __forceinline__ int32_t to_fixed(float v, float fixed) {
    const float q = rintf(v * fixed);
    return q >= 2147483648.0f ? 2147483647 : q <= -2147483648.0f ? -2147483647 : (int32_t)(q != q ? 0.0f : q);
}

// What a gradient's sums become: a row of `type`, written or added to.
struct Gradient {
    void* out;
    uint64_t ld;
    uint32_t type;  // hc_type
    uint32_t accumulate;
    float fixed;
    float unit;     // of a product with an fp16 dz: what its sums are multiplied by
};

template <typename T>
__device__ __forceinline__ void store_gradient_as(const Gradient& g, uint64_t row, uint32_t col,
                                                  uint32_t count, float (&v)[8]) {
    T* p = static_cast<T*>(g.out) + row * g.ld + col;
    if (g.accumulate) {
        float old[8];
        load8(p, count, old);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += old[e];
    }
    store8(p, count, v);
}

__device__ __forceinline__ void store_gradient(const Gradient& g, uint64_t row, uint32_t col,
                                               uint32_t count, float (&v)[8]) {
    switch (g.type) {
        case HC_T_F32: store_gradient_as<float>(g, row, col, count, v); break;
        case HC_T_BF16: store_gradient_as<__bf16>(g, row, col, count, v); break;
        case HC_T_F16: store_gradient_as<_Float16>(g, row, col, count, v); break;
        default: {
            int32_t* p = static_cast<int32_t*>(g.out) + row * g.ld + col;
#pragma unroll
            for (int e = 0; e < 8; e++)
                if ((uint32_t)e < count) {
                    int64_t q = to_fixed(v[e], g.fixed);
                    if (g.accumulate) {
                        q += p[e];
                        q = q > 2147483647 ? 2147483647 : q < -2147483647 ? -2147483647 : q;
                    }
                    p[e] = (int32_t)q;
                }
        }
    }
}

}  // namespace hc
