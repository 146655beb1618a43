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

template <int PT>
__device__ __forceinline__ float ld_val(const void* p, uint64_t i) {
    if (PT == PT_FP32) return static_cast<const float*>(p)[i];
    const uint16_t h = static_cast<const uint16_t*>(p)[i];
    if (PT == PT_BF16) return __uint_as_float((uint32_t)h << 16);
    return (float)__builtin_bit_cast(_Float16, h);
}
template <int PT>
__device__ __forceinline__ void st_val(void* p, uint64_t i, float x) {
    if (PT == PT_FP32) static_cast<float*>(p)[i] = x;
    else if (PT == PT_BF16) static_cast<__bf16*>(p)[i] = (__bf16)x;
    else static_cast<_Float16*>(p)[i] = (_Float16)x;
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

__device__ __forceinline__ float from_e4m3(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }
__device__ __forceinline__ float from_e5m2(uint8_t c) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(c << 8)); }

// float8 code of y in 0..TOP: the leading bits of the fp32 number, or for a float8
// subnormal those of the number plus the smallest normal one (whose last place is the
// subnormals' step), after adding a noise below the last place.
template <int MAN, int BIAS>
__device__ __forceinline__ uint32_t to_float8(float y, uint32_t noise16) {
    constexpr int DROP = 23 - MAN;
    const float lowest = __uint_as_float((uint32_t)(128 - BIAS) << 23);   // 2^(1 - BIAS)
    const bool small = y < lowest;
    const uint32_t at = __float_as_uint(small ? y + lowest : y);
    const uint32_t up = (at + (noise16 << (DROP - 16)) + (1u << (DROP - 17))) >> DROP;
    return up - ((uint32_t)(small ? 128 - BIAS : 127 - BIAS) << MAN);
}

constexpr float E4M3_TOP = 448.f, E5M2_TOP = 57344.f;
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

template <int PT, int GT, bool S8>
__global__ void __launch_bounds__(256) k_adamw(AdamwArgs a) {
#pragma clang fp contract(off)
    // no fused multiply-adds: the 8-bit codes are a function of separately rounded operations
    const int k = adamw_tensor(a);
    const AdamwTensor T = a.t[k];
    const uint32_t t = (uint32_t)*a.step + 1u;
    const float c1 = (float)(1.0 - power(a.beta1, t)), c2 = (float)(1.0 - power(a.beta2, t));
    const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
    const float flr = (float)lr, decay = (float)(lr * a.decay), eps = (float)a.eps;
    const float b1 = (float)a.beta1, b2 = (float)a.beta2, d1 = (float)(1.0 - a.beta1), d2 = (float)(1.0 - a.beta2);
    const uint64_t lo = (uint64_t)(blockIdx.x - a.wg_begin[k]) * ADAMW_CHUNK;
    __shared__ uint32_t top[2][4];
    for (uint64_t i = lo + threadIdx.x; i < lo + ADAMW_CHUNK; i += 256) {
        const bool in = i < T.n;
        float m = 0.f, v = 0.f;
        if (in) {
            const float g = ld_val<GT>(T.g, i);
            if (S8) {
                m = from_e4m3(static_cast<const uint8_t*>(T.m)[i]) * T.m_scale[i / ADAMW_BLOCK];
                v = from_e5m2(static_cast<const uint8_t*>(T.v)[i]) * T.v_scale[i / ADAMW_BLOCK];
            } else {
                m = static_cast<const float*>(T.m)[i];
                v = static_cast<const float*>(T.v)[i];
            }
            m = m * b1 + g * d1;
            v = v * b2 + g * g * d2;
            float p = T.master ? T.master[i] : ld_val<PT>(T.p, i);
            p = p - p * decay - flr * (m / c1) / (sqrtf(v / c2) + eps);
            if (T.master) T.master[i] = p;
            st_val<PT>(T.p, i, p);
            if (!S8) {
                static_cast<float*>(T.m)[i] = m;
                static_cast<float*>(T.v)[i] = v;
            }
        }
        if (S8) {
            // the block's largest magnitudes, as bit patterns: Inf and NaN are above all
            uint32_t am = __float_as_uint(m) & 0x7FFFFFFFu, av = __float_as_uint(v) & 0x7FFFFFFFu;
            for (int o = 32; o; o >>= 1) {
                am = max(am, (uint32_t)__shfl_xor((int)am, o));
                av = max(av, (uint32_t)__shfl_xor((int)av, o));
            }
            __syncthreads();
            if ((threadIdx.x & 63) == 0) {
                top[0][threadIdx.x >> 6] = am;
                top[1][threadIdx.x >> 6] = av;
            }
            __syncthreads();
            am = max(max(top[0][0], top[0][1]), max(top[0][2], top[0][3]));
            av = max(max(top[1][0], top[1][1]), max(top[1][2], top[1][3]));
            const float fm = __uint_as_float(am), fv = __uint_as_float(av);
            const uint32_t h = hash32((uint32_t)(i >> 1) + t * 0x9E3779B9u + a.seed);
            const uint32_t noise = (i & 1) ? h >> 16 : h & 0xFFFFu;
            const float ym = fminf(fabsf(m) * (fm >= SCALE_LIVE ? (1.0f / fm) * E4M3_TOP : 0.f), E4M3_TOP);
            const float yv = fminf(fabsf(v) * (fv >= SCALE_LIVE ? (1.0f / fv) * E5M2_TOP : 0.f), E5M2_TOP);
            uint32_t cm = to_float8<3, 7>(ym, noise), cv = to_float8<2, 15>(yv, noise);
            if (cv == 0 && yv > 0.f) cv = 1;
            if (m < 0.f && cm) cm |= 0x80u;
            if (in) {
                static_cast<uint8_t*>(T.m)[i] = (uint8_t)cm;
                static_cast<uint8_t*>(T.v)[i] = (uint8_t)cv;
            }
            if (in && threadIdx.x == 0) {
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
