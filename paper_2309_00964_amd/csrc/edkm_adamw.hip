// AdamW over many tensors in one launch, for gfx950 (MI355X).
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   p = p - lr decay p - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
//
// with m and v as fp32, or as float8 numbers with an fp32 scale per 256 elements.

#include "edkm_layer.h"

#include <hip/hip_fp16.h>

namespace edkm {

typedef __attribute__((ext_vector_type(2))) float f32x2;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

template <int PT>
__device__ __forceinline__ float value_of(uint32_t h) {
    if (PT == PT_BF16) return __uint_as_float(h << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}
template <int PT>
__device__ __forceinline__ uint16_t bits_of(float x) {
    if (PT == PT_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// Eight elements from i on; `vec`: all there, on a boundary of their size.  Elements past n
// are zeros, and not written.
template <int PT>
__device__ __forceinline__ void load8(const void* p, uint64_t i, uint64_t n, bool vec, float (&x)[8]) {
    if (vec) {
        if (PT == PT_FP32) {
            const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i));
            const f32x4 b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i) + 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = a[j];
                x[j + 4] = b[j];
            }
        } else {
            const u32x4 a = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i));
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = value_of<PT>(j & 1 ? a[j / 2] >> 16 : a[j / 2] & 0xFFFFu);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = 0.f;
            if (i + j < n) x[j] = PT == PT_FP32 ? static_cast<const float*>(p)[i + j] : value_of<PT>(static_cast<const uint16_t*>(p)[i + j]);
        }
    }
}
template <int PT>
__device__ __forceinline__ void store8(void* p, uint64_t i, uint64_t n, bool vec, const float (&x)[8]) {
    if (vec) {
        if (PT == PT_FP32) {
            f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + i);
            __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, q);
            __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, q + 1);
        } else {
            u32x4 a;
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = bits_of<PT>(x[2 * j]) | ((uint32_t)bits_of<PT>(x[2 * j + 1]) << 16);
            __builtin_nontemporal_store(a, reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + i));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < n) {
                if (PT == PT_FP32) static_cast<float*>(p)[i + j] = x[j];
                else static_cast<uint16_t*>(p)[i + j] = bits_of<PT>(x[j]);
            }
    }
}
__device__ __forceinline__ u32x2 load_codes(const void* p, uint64_t i, uint64_t n, bool vec) {
    const uint8_t* q = static_cast<const uint8_t*>(p) + i;
    if (vec) return __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(q));
    u32x2 c = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (i + j < n) c[j / 4] |= (uint32_t)q[j] << (8 * (j & 3));
    return c;
}
__device__ __forceinline__ void store_codes(void* p, uint64_t i, uint64_t n, bool vec, u32x2 c) {
    uint8_t* q = static_cast<uint8_t*>(p) + i;
    if (vec) {
        __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(q));
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (i + j < n) q[j] = (uint8_t)(c[j / 4] >> (8 * (j & 3)));
}

// A 32-bit hash (MurmurHash3's finaliser, A. Appleby): the rounding noise of a pair
// of elements.
__device__ __forceinline__ uint32_t hash32(uint32_t h) {
    h ^= h >> 16;
    h *= 0x85EBCA6Bu;
    h ^= h >> 13;
    h *= 0xC2B2AE35u;
    return h ^ (h >> 16);
}

constexpr float E4M3_TOP = 448.f, E5M2_TOP = 57344.f, E5M2_LEAST = 0x1p-16f;
constexpr float SCALE_LIVE = 0x1p-100f;   // blocks below it are stored as zeros

// beta^t, t >= 0
__device__ __forceinline__ double power(double beta, uint32_t t) {
    double r = 1.0;
    for (; t; t >>= 1, beta *= beta)
        if (t & 1) r *= beta;
    return r;
}

__device__ __forceinline__ int adamw_tensor(const AdamwArgs& a) {
    int k = 0;
    for (int i = 1; i < MAXB; ++i) k += blockIdx.x >= a.wg_begin[i];
    return k;
}

// the largest of 32 lanes (a half wave), in all of them
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t half_max(uint32_t x) {
    x = max(x, dpp<0x121>(x));   // rotations by 1, 2, 4, 8 within rows of sixteen
    x = max(x, dpp<0x122>(x));
    x = max(x, dpp<0x124>(x));
    x = max(x, dpp<0x128>(x));
    return max(x, (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x401F));   // lane ^ 16
}

// Eight elements per thread and pass, 32 lanes for the 256 elements of a scale.  Bound by
// the bytes moved (10.06 B per bf16 element with 8-bit states, 22 with fp32 ones) and, in the
// 8-bit form, as much by its arithmetic, which keeps the vector units busy for 85% of the time
// (14% with fp32 states).  The 202M bf16 weights of a decoder layer take 374 to 382 us with
// 8-bit states (5.4 TB/s; an elementwise kernel that reads as much as it writes reaches 6.2),
// 658 with fp32 masters, 924 with fp32 states (4.8 TB/s) and 1199 with both.
template <int PT, int GT, bool S8>
__global__ void __launch_bounds__(256) k_adamw(AdamwArgs a) {
#pragma clang fp contract(off)
    // no fused multiply-adds: m, v and their codes are a function of separately rounded operations
    const int k = adamw_tensor(a);
    const AdamwTensor T = a.t[k];
    const uint32_t t = (uint32_t)*a.step + 1u;
    const float i1 = (float)(1.0 / (1.0 - power(a.beta1, t))), i2 = (float)(1.0 / (1.0 - power(a.beta2, t)));
    const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
    const float step1 = (float)lr * i1, decay = (float)(lr * a.decay), eps = (float)a.eps;
    const float b1 = (float)a.beta1, b2 = (float)a.beta2, d1 = (float)(1.0 - a.beta1), d2 = (float)(1.0 - a.beta2);
    const uint64_t lo = (uint64_t)(blockIdx.x - a.wg_begin[k]) * a.chunk, hi = min(lo + a.chunk, T.n);
    const uint32_t key = t * 0x9E3779B9u + a.seed;
    // whole blocks of 256 elements, so that all lanes of a block's 32 take part in its maximum
    const uint64_t end = S8 ? (hi + ADAMW_BLOCK - 1) & ~(uint64_t)(ADAMW_BLOCK - 1) : hi;
    for (uint64_t i = lo + threadIdx.x * 8; i < end; i += 2048) {
        const bool vec = a.aligned && i + 8 <= T.n;
        float g[8], p[8], m[8], v[8];
        load8<GT>(T.g, i, T.n, vec, g);
        if (T.master) load8<PT_FP32>(T.master, i, T.n, vec, p);
        else load8<PT>(T.p, i, T.n, vec, p);
        if (S8) {
            const u32x2 cm = load_codes(T.m, i, T.n, vec), cv = load_codes(T.v, i, T.n, vec);
            const float sm = T.m_scale[i / ADAMW_BLOCK], sv = T.v_scale[i / ADAMW_BLOCK];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm[h], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm[h], true);
                const f32x2 v0 = __builtin_amdgcn_cvt_pk_f32_bf8((int)cv[h], false), v1 = __builtin_amdgcn_cvt_pk_f32_bf8((int)cv[h], true);
                m[4 * h] = m0[0] * sm, m[4 * h + 1] = m0[1] * sm, m[4 * h + 2] = m1[0] * sm, m[4 * h + 3] = m1[1] * sm;
                v[4 * h] = v0[0] * sv, v[4 * h + 1] = v0[1] * sv, v[4 * h + 2] = v1[0] * sv, v[4 * h + 3] = v1[1] * sv;
            }
        } else {
            load8<PT_FP32>(T.m, i, T.n, vec, m);
            load8<PT_FP32>(T.v, i, T.n, vec, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = m[j] * b1 + g[j] * d1;
            v[j] = v[j] * b2 + g[j] * g[j] * d2;
            // Square root and reciprocal are the hardware's estimates (an ulp each): they reach p
            // only, whose update they move by less than its own rounding.  The root's takes no
            // subnormals; 2^-126 more changes nothing above 2^-102.
            const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(__builtin_fmaf(v[j], i2, 0x1p-126f)) + eps);
            p[j] = __builtin_fmaf(m[j] * -step1, r, __builtin_fmaf(p[j], -decay, p[j]));
        }
        if (T.master) store8<PT_FP32>(T.master, i, T.n, vec, p);
        store8<PT>(T.p, i, T.n, vec, p);
        if (!S8) {
            store8<PT_FP32>(T.m, i, T.n, vec, m);
            store8<PT_FP32>(T.v, i, T.n, vec, v);
        } else {
            // the block's largest magnitudes, as bit patterns: Inf and NaN are above all
            uint32_t am = 0, av = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (!vec && i + j >= T.n) m[j] = v[j] = 0.f;
                am = max(am, __float_as_uint(m[j]) & 0x7FFFFFFFu);
                av = max(av, __float_as_uint(v[j]) & 0x7FFFFFFFu);
            }
            am = half_max(am);
            av = half_max(av);
            const float fm = __uint_as_float(am), fv = __uint_as_float(av);
            const float im = fm >= SCALE_LIVE ? (1.0f / fm) * E4M3_TOP : 0.f, iv = fv >= SCALE_LIVE ? (1.0f / fv) * E5M2_TOP : 0.f;
            // The conversions' noise is added below the last place that they keep, in units of
            // its 2^-32: sixteen bits of the hash and a half of their last place.
            u32x2 cm = {0, 0}, cv = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const uint32_t h = hash32((uint32_t)((i + j) >> 1) + key);
                const int n0 = (int)((h << 16) | 0x8000u), n1 = (int)((h & 0xFFFF0000u) | 0x8000u);
                const float x0 = __builtin_amdgcn_fmed3f(m[j] * im, -E4M3_TOP, E4M3_TOP);
                const float x1 = __builtin_amdgcn_fmed3f(m[j + 1] * im, -E4M3_TOP, E4M3_TOP);
                // a second moment above 0 is kept at the smallest e5m2 number at least
                float y0 = v[j] * iv, y1 = v[j + 1] * iv;
                y0 = y0 > 0.f ? __builtin_amdgcn_fmed3f(y0, E5M2_LEAST, E5M2_TOP) : 0.f;
                y1 = y1 > 0.f ? __builtin_amdgcn_fmed3f(y1, E5M2_LEAST, E5M2_TOP) : 0.f;
                if (j & 2) {
                    cm[j / 4] = __builtin_amdgcn_cvt_sr_fp8_f32(x0, n0, (int)cm[j / 4], 2);
                    cm[j / 4] = __builtin_amdgcn_cvt_sr_fp8_f32(x1, n1, (int)cm[j / 4], 3);
                    cv[j / 4] = __builtin_amdgcn_cvt_sr_bf8_f32(y0, n0, (int)cv[j / 4], 2);
                    cv[j / 4] = __builtin_amdgcn_cvt_sr_bf8_f32(y1, n1, (int)cv[j / 4], 3);
                } else {
                    cm[j / 4] = __builtin_amdgcn_cvt_sr_fp8_f32(x0, n0, (int)cm[j / 4], 0);
                    cm[j / 4] = __builtin_amdgcn_cvt_sr_fp8_f32(x1, n1, (int)cm[j / 4], 1);
                    cv[j / 4] = __builtin_amdgcn_cvt_sr_bf8_f32(y0, n0, (int)cv[j / 4], 0);
                    cv[j / 4] = __builtin_amdgcn_cvt_sr_bf8_f32(y1, n1, (int)cv[j / 4], 1);
                }
            }
            store_codes(T.m, i, T.n, vec, cm);
            store_codes(T.v, i, T.n, vec, cv);
            if ((threadIdx.x & 31) == 0 && i < T.n) {
                // a block with an Inf or NaN decodes to NaN throughout
                T.m_scale[i / ADAMW_BLOCK] = am >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : fm >= SCALE_LIVE ? fm * (1.0f / E4M3_TOP) : 0.f;
                T.v_scale[i / ADAMW_BLOCK] = av >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : fv >= SCALE_LIVE ? fv * (1.0f / E5M2_TOP) : 0.f;
            }
        }
    }
}

__global__ void k_adamw_tick(int32_t* step) { *step += 1; }

#define EDKM_GO(kern, grid, block, ...)                       \
    do {                                                       \
        hipLaunchKernelGGL(kern, grid, block, 0, s, __VA_ARGS__); \
        const hipError_t e_ = hipGetLastError();               \
        if (e_ != hipSuccess) return e_;                       \
    } while (0)

template <int PT, int GT>
static hipError_t adamw_pg(const AdamwArgs& a, uint32_t grid, int bits, hipStream_t s) {
    if (bits == 8) EDKM_GO((k_adamw<PT, GT, true>), dim3(grid), dim3(256), a);
    else EDKM_GO((k_adamw<PT, GT, false>), dim3(grid), dim3(256), a);
    return hipSuccess;
}

hipError_t launch_adamw(const AdamwArgs& a, uint32_t grid, int pt, int gt, int bits, hipStream_t s) {
    if (pt == PT_FP32) return adamw_pg<PT_FP32, PT_FP32>(a, grid, bits, s);
    if (pt == PT_BF16)
        return gt == PT_FP32 ? adamw_pg<PT_BF16, PT_FP32>(a, grid, bits, s) : adamw_pg<PT_BF16, PT_BF16>(a, grid, bits, s);
    return gt == PT_FP32 ? adamw_pg<PT_FP16, PT_FP32>(a, grid, bits, s) : adamw_pg<PT_FP16, PT_FP16>(a, grid, bits, s);
}

hipError_t launch_adamw_tick(int32_t* step, hipStream_t s) {
    EDKM_GO(k_adamw_tick, dim3(1), dim3(1), step);
    return hipSuccess;
}

}  // namespace edkm
