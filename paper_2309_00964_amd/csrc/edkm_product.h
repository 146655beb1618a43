// Device code that the products share: the two 16-bit formats, activations, palettes.
#pragma once
#include "edkm_layer.h"

#include <hip/hip_fp16.h>

namespace edkm {

typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
struct __attribute__((packed)) S16x8 { s16x8 v; };   // at any address

// ----------------------------------------------------------------------------
// the two 16-bit formats

template <int F>
__device__ __forceinline__ float to_f32(uint16_t h) {
    if (F == FMT_BF16) return __uint_as_float((uint32_t)h << 16);
    return (float)__builtin_bit_cast(_Float16, h);
}
// to nearest even; NaN stays NaN
template <int F>
__device__ __forceinline__ uint16_t to_16(float x) {
    if (F == FMT_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    return __builtin_bit_cast(uint16_t, (_Float16)x);
}
template <int F>
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
    if constexpr (F == FMT_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// ----------------------------------------------------------------------------
// activations and their derivatives

// e^-u for u >= 0 or any sign: the hardware's 2^x (an ulp) on a rounded product; the
// relative error |u| 2^-23 stays far below the 16-bit results' rounding wherever the
// result is not negligible.
__device__ __forceinline__ float exp_minus(float u) { return __builtin_amdgcn_exp2f(u * -1.4426950408889634f); }
// 1 / (1 + e^-z)
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + exp_minus(z)); }
// The normal distribution's Phi(z) and e^(-z^2 / 2), which its tail is a polynomial times:
// Phi(-|z|) = e^(-x^2) t Q(t) with x = |z| / sqrt 2 and t = 1 / (1 + 0.51 x), the form of
// Abramowitz and Stegun's 7.1.26, whose tail is off by 0.4% at z = -4 and 4% at -13.  Q here is
// of degree 6 and has the least relative error over x <= 9.5 (7.3e-7; a linear programme over
// Chebyshev points), so that z Phi(z) keeps its leading digits for negative z too.  With fp32's
// roundings, mostly the exponent's, Phi is off by 1e-6 at z = -1, 5e-6 at -6 and 2e-5 at -13,
// relative; half a step of fp16 is 5e-4.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(fmaf(0.51f, x, 1.0f));
    e = exp_minus(x * x);
    float q = fmaf(t, 0.0476253042f, -0.180841452f);
    q = fmaf(t, q, 0.180943695f);
    q = fmaf(t, q, 0.0263486397f);
    q = fmaf(t, q, 0.139961549f);
    q = fmaf(t, q, 0.141998004f);
    q = fmaf(t, q, 0.143964306f);
    const float tail = e * t * q;
    return z < 0.f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float act_value(float z, int act) {
    float e;
    switch (act) {
    case ACT_RELU: return z < 0.f ? 0.f : z;
    case ACT_GELU: return z * normal_cdf(z, e);
    case ACT_SILU: return z * logistic(z);
    default: return z;
    }
}
__device__ __forceinline__ float act_slope(float z, int act) {
    switch (act) {
    case ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case ACT_GELU: {
        float e;
        const float p = normal_cdf(z, e);
        return fmaf(z * 0.39894228040143268f, e, p);
    }
    case ACT_SILU: {
        const float q = logistic(z);
        return q * fmaf(z, 1.0f - q, 1.0f);
    }
    default: return 1.f;
    }
}

// The pre-activation as it is kept for the backward pass.  A finite z that the format
// cannot hold takes its largest value: every activation's slope is constant out there,
// while at an infinity gelu's and silu's formulas give NaN.
template <int F>
__device__ __forceinline__ uint16_t keep_z(float z) {
    const uint16_t h = to_16<F>(z);
    const uint16_t top = F == FMT_BF16 ? 0x7F7F : 0x7BFF;
    if ((h & 0x7FFF) == top + 1 && __builtin_isfinite(z)) return (h & 0x8000) | top;
    return h;
}

// ----------------------------------------------------------------------------
// palettes

struct __attribute__((packed)) U64 { uint64_t v; };
struct __attribute__((packed)) U32 { uint32_t v; };

// Table of pairs: entry e holds the values of indices e mod 2^b and e / 2^b, once per LDS
// bank, so that the lanes of a wave look up without conflicts.
constexpr int PAIR_BANKS = 32;

// The 8 b bits of eight consecutive indices, from index i on, in the low bits.  Reads
// nothing past the last byte.
__device__ __forceinline__ uint32_t load_idx8(const uint8_t* idx, uint64_t nbytes, uint64_t i, int bits) {
    const uint64_t o = i * (uint64_t)bits;
    const uint64_t at = o >> 3;
    uint64_t v = 0;
    if (at + 8 <= nbytes) {
        v = reinterpret_cast<const U64*>(idx + at)->v;
    } else {
        for (int j = 0; j < 8; ++j)
            if (at + j < nbytes) v |= (uint64_t)idx[at + j] << (8 * j);
    }
    return (uint32_t)(v >> (o & 7));
}

// Table lookups in registers: the low and the high bytes of up to sixteen 16-bit values in
// four registers each; v_perm_b32 picks four bytes of two registers at once.
template <int F>
struct Decoder {
    uint32_t lo[4], hi[4];

    __device__ __forceinline__ void init(const float* lut, int bits) {
        const int k = 1 << bits;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = hi[i] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i * 4 + j < k) {
                    const uint32_t h = to_16<F>(lut[i * 4 + j]);
                    lo[i] |= (h & 255) << (8 * j);
                    hi[i] |= (h >> 8) << (8 * j);
                }
        }
    }
    // four values for the four indices in sel's bytes: two registers of two
    __device__ __forceinline__ void four(uint32_t sel, bool wide, uint32_t& v01, uint32_t& v23) const {
        uint32_t l, h;
        if (wide) {       // sixteen entries: both halves, then the one that bit 3 names
            const uint32_t s = sel & 0x07070707u, up = sel & 0x08080808u, mask = (up << 5) - (up >> 3);
            const uint32_t l0 = __builtin_amdgcn_perm(lo[1], lo[0], s), l1 = __builtin_amdgcn_perm(lo[3], lo[2], s);
            const uint32_t h0 = __builtin_amdgcn_perm(hi[1], hi[0], s), h1 = __builtin_amdgcn_perm(hi[3], hi[2], s);
            l = (l1 & mask) | (l0 & ~mask);
            h = (h1 & mask) | (h0 & ~mask);
        } else {
            l = __builtin_amdgcn_perm(lo[1], lo[0], sel);
            h = __builtin_amdgcn_perm(hi[1], hi[0], sel);
        }
        v01 = __builtin_amdgcn_perm(h, l, 0x05010400u);
        v23 = __builtin_amdgcn_perm(h, l, 0x07030602u);
    }
    // the values of eight packed indices
    __device__ __forceinline__ s16x8 eight(uint32_t w, int bits) const {
        typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
        uint32_t s0, s1;
        if (bits == 4) {
            s0 = spread(w & 0xFFFFu, 4);
            s1 = spread(w >> 16, 4);
        } else {
            s0 = spread(w & ((1u << (4 * bits)) - 1), bits);
            s1 = spread((w >> (4 * bits)) & ((1u << (4 * bits)) - 1), bits);
        }
        u32x4 v;
        uint32_t a, b;
        four(s0, bits == 4, a, b);
        v[0] = a;
        v[1] = b;
        four(s1, bits == 4, a, b);
        v[2] = a;
        v[3] = b;
        return __builtin_bit_cast(s16x8, v);
    }
    // 4 b bits into the low bits of four bytes
    __device__ __forceinline__ static uint32_t spread(uint32_t x, int b) {
        x = (x | (x << (16 - 2 * b))) & (((1u << (2 * b)) - 1) * 0x10001u);
        return (x | (x << (8 - b))) & (((1u << b) - 1) * 0x01010101u);
    }
};

// eight consecutive values, `left` of them there (zeros after them)
template <bool PAST = false>
__device__ __forceinline__ s16x8 row8(const uint16_t* q, int left) {
    typedef short any8 __attribute__((ext_vector_type(8), aligned(2)));
    if (left >= 8) return PAST ? __builtin_nontemporal_load(reinterpret_cast<const any8*>(q)) : reinterpret_cast<const S16x8*>(q)->v;
    s16x8 v = {};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) v[j] = (short)q[j];
    return v;
}

// the first `n` of eight values, zeros after them
__device__ __forceinline__ s16x8 keep_first(s16x8 v, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j >= n) v[j] = 0;
    return v;
}

// A one-dimensional grid of any number of workgroups, whose kernel starts with args.first
#define EDKM_GO_PARTS(kern, groups, threads, args, ...)                                                          \
    do {                                                                                                          \
        const hipError_t p_ = in_parts((groups), (threads), hipSuccess, [&](uint32_t first_, uint32_t groups_) {  \
            (args).first = first_;                                                                                \
            hipLaunchKernelGGL(kern, dim3(groups_), dim3(threads), 0, s, args, ##__VA_ARGS__);                    \
            return hipGetLastError();                                                                             \
        });                                                                                                       \
        if (p_ != hipSuccess) return p_;                                                                          \
    } while (0)

#define EDKM_GO(kern, grid, block, ...)                       \
    do {                                                       \
        hipLaunchKernelGGL(kern, grid, block, 0, s, __VA_ARGS__); \
        const hipError_t e_ = hipGetLastError();               \
        if (e_ != hipSuccess) return e_;                       \
    } while (0)


}  // namespace edkm
