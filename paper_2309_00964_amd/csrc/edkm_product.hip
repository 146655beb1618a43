// Products with an epilogue for gfx950 (MI355X): y = act(x W^T + bias) + residual with
// 16-bit or palettized weights, the products of its backward pass, and the 16-bit
// weights of a palette.

#include "edkm_layer.h"

#include <hip/hip_fp16.h>

namespace edkm {

typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

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

__device__ __forceinline__ float act_value(float z, int act) {
    switch (act) {
    case ACT_RELU: return z < 0.f ? 0.f : z;
    case ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    case ACT_SILU: return z / (1.0f + expf(-z));
    default: return z;
    }
}
__device__ __forceinline__ float act_slope(float z, int act) {
    switch (act) {
    case ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case ACT_GELU:
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    case ACT_SILU: {
        const float q = 1.0f / (1.0f + expf(-z));
        return q * (1.0f + z * (1.0f - q));
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

template <int F>
__global__ void __launch_bounds__(256) k_unpalettize(const uint8_t* idx, uint64_t nbytes, uint64_t n, int bits,
                                                     const float* lut, uint16_t* out) {
    __shared__ uint16_t tab[KMAX];
    if (threadIdx.x < (1u << bits)) tab[threadIdx.x] = to_16<F>(lut[threadIdx.x]);
    __syncthreads();
    const uint64_t i = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= n) return;
    const uint32_t w = load_idx8(idx, nbytes, i, bits);
    for (int j = 0; j < 8; ++j)
        if (i + j < n) out[i + j] = tab[(w >> (j * bits)) & ((1u << bits) - 1)];
}

// ----------------------------------------------------------------------------
// products

constexpr int TM = 64, TN = 64, TK = 32, TPAD = 8;

// Eight consecutive depths of one row; zeros past the ends.
template <int F, int OP>
__device__ __forceinline__ s16x8 load8(const ProductArgs& p, const uint16_t* m, int64_t ld, int row, int nrow, int d,
                                       const uint16_t* tab) {
    s16x8 v = {};
    if (row >= nrow || d >= p.depth) return v;
    const int left = p.depth - d;
    if (OP == OP_ROWS) {
        const uint16_t* s = m + (int64_t)row * ld + d;
        for (int j = 0; j < 8; ++j)
            if (j < left) v[j] = (short)s[j];
    } else if (OP == OP_DEPTH) {
        const uint16_t* s = m + (int64_t)d * ld + row;
        for (int j = 0; j < 8; ++j)
            if (j < left) v[j] = (short)s[(int64_t)j * ld];
    } else {
        const uint32_t w = load_idx8(p.idx, p.idx_bytes, (uint64_t)row * (uint64_t)p.depth + d, p.bits);
        for (int j = 0; j < 8; ++j)
            if (j < left) v[j] = (short)tab[(w >> (j * p.bits)) & ((1u << p.bits) - 1)];
    }
    return v;
}

template <int F, int OPA, int OPB>
__global__ void __launch_bounds__(256) k_product(ProductArgs p) {
    __shared__ __attribute__((aligned(16))) uint16_t la[TM][TK + TPAD], lb[TN][TK + TPAD];
    __shared__ uint16_t tab[KMAX];
    if (OPB == OP_PALETTE && threadIdx.x < (1u << p.bits)) tab[threadIdx.x] = to_16<F>(p.lut[threadIdx.x]);
    __syncthreads();
    const int r0 = blockIdx.y * TM, c0 = blockIdx.x * TN;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wr = (wave >> 1) * 32, wc = (wave & 1) * 32;
    const int srow = OPA == OP_ROWS ? threadIdx.x >> 2 : threadIdx.x & 63;
    const int sd = (OPA == OP_ROWS ? threadIdx.x & 3 : threadIdx.x >> 6) * 8;
    const int trow = OPB != OP_DEPTH ? threadIdx.x >> 2 : threadIdx.x & 63;
    const int td = (OPB != OP_DEPTH ? threadIdx.x & 3 : threadIdx.x >> 6) * 8;
    f32x4 acc[2][2] = {};
    for (int d0 = 0; d0 < p.depth; d0 += TK) {
        const s16x8 va = load8<F, OPA>(p, p.a, p.lda, r0 + srow, p.rows, d0 + sd, tab);
        const s16x8 vb = load8<F, OPB>(p, p.b, p.ldb, c0 + trow, p.cols, d0 + td, tab);
        __syncthreads();
        *reinterpret_cast<s16x8*>(&la[srow][sd]) = va;
        *reinterpret_cast<s16x8*>(&lb[trow][td]) = vb;
        __syncthreads();
        const int l = lane & 15, g = (lane >> 4) * 8;
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j)
                acc[i][j] = mfma16<F>(*reinterpret_cast<s16x8*>(&lb[wc + 16 * j + l][g]),
                                      *reinterpret_cast<s16x8*>(&la[wr + 16 * i + l][g]), acc[i][j]);
    }
    for (int i = 0; i < 2; ++i) {
        const int r = r0 + wr + 16 * i + (lane & 15);
        if (r >= p.rows) continue;
        for (int j = 0; j < 2; ++j)
            for (int q = 0; q < 4; ++q) {
                const int c = c0 + wc + 16 * j + (lane >> 4) * 4 + q;
                if (c >= p.cols) continue;
                float z = acc[i][j][q];
                if (p.bias) z += to_f32<F>(p.bias[c]);
                if (p.z) p.z[(int64_t)r * p.cols + c] = keep_z<F>(z);
                float y = act_value(z, p.act);
                if (p.res) y += to_f32<F>(p.res[(int64_t)r * p.ldr + c]);
                p.out[(int64_t)r * p.ldo + c] = to_16<F>(y);
            }
    }
}

template <int F>
__global__ void __launch_bounds__(256) k_dz(DzArgs a) {
    __shared__ float red[4][DZ_COLS];
    const int c = blockIdx.x * DZ_COLS + (threadIdx.x & 63), q = threadIdx.x >> 6;
    const int r0 = blockIdx.y * DZ_ROWS, r1 = min(r0 + DZ_ROWS, a.rows);
    float sum = 0.f;
    if (c < a.cols)
        for (int r = r0 + q; r < r1; r += 4) {
            float d = to_f32<F>(a.dy[(int64_t)r * a.lddy + c]);
            if (a.act != ACT_NONE) {
                d *= act_slope(to_f32<F>(a.z[(int64_t)r * a.cols + c]), a.act);
                a.dz[(int64_t)r * a.cols + c] = to_16<F>(d);
            }
            sum += d;
        }
    red[q][threadIdx.x & 63] = sum;
    __syncthreads();
    if (a.dbias && q == 0 && c < a.cols)
        a.part[(int64_t)blockIdx.y * a.cols + c] =
            (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
}

template <int F>
__global__ void __launch_bounds__(256) k_dbias(DzArgs a, int chunks) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float sum = 0.f;
    for (int i = 0; i < chunks; ++i) sum += a.part[(int64_t)i * a.cols + c];
    a.dbias[c] = to_16<F>(sum);
}

// ----------------------------------------------------------------------------
// launches

#define EDKM_GO(kern, grid, block, ...)                       \
    do {                                                       \
        hipLaunchKernelGGL(kern, grid, block, 0, s, __VA_ARGS__); \
        const hipError_t e_ = hipGetLastError();               \
        if (e_ != hipSuccess) return e_;                       \
    } while (0)

template <int F>
static hipError_t product_f(const ProductArgs& p, int opa, int opb, hipStream_t s) {
    const dim3 grid((p.cols + TN - 1) / TN, (p.rows + TM - 1) / TM);
    if (opa == OP_ROWS && opb == OP_ROWS) EDKM_GO((k_product<F, OP_ROWS, OP_ROWS>), grid, dim3(256), p);
    else if (opa == OP_ROWS && opb == OP_DEPTH) EDKM_GO((k_product<F, OP_ROWS, OP_DEPTH>), grid, dim3(256), p);
    else if (opa == OP_DEPTH && opb == OP_DEPTH) EDKM_GO((k_product<F, OP_DEPTH, OP_DEPTH>), grid, dim3(256), p);
    else EDKM_GO((k_product<F, OP_ROWS, OP_PALETTE>), grid, dim3(256), p);
    return hipSuccess;
}

hipError_t launch_product(const ProductArgs& p, int fmt, int opa, int opb, hipStream_t s) {
    return fmt == FMT_BF16 ? product_f<FMT_BF16>(p, opa, opb, s) : product_f<FMT_FP16>(p, opa, opb, s);
}

template <int F>
static hipError_t dz_f(const DzArgs& a, hipStream_t s) {
    const int chunks = (a.rows + DZ_ROWS - 1) / DZ_ROWS;
    if (chunks > 0 && (a.dbias || a.act != ACT_NONE))
        EDKM_GO(k_dz<F>, dim3((a.cols + DZ_COLS - 1) / DZ_COLS, chunks), dim3(256), a);
    if (a.dbias) EDKM_GO(k_dbias<F>, dim3((a.cols + 255) / 256), dim3(256), a, chunks);
    return hipSuccess;
}

hipError_t launch_dz(const DzArgs& a, int fmt, hipStream_t s) {
    return fmt == FMT_BF16 ? dz_f<FMT_BF16>(a, s) : dz_f<FMT_FP16>(a, s);
}

hipError_t launch_unpalettize(const uint8_t* idx, uint64_t idx_bytes, uint64_t n, int bits, int fmt, const float* lut,
                              uint16_t* out, hipStream_t s) {
    const dim3 grid((uint32_t)((n + 2047) / 2048));
    if (fmt == FMT_BF16) EDKM_GO(k_unpalettize<FMT_BF16>, grid, dim3(256), idx, idx_bytes, n, bits, lut, out);
    else EDKM_GO(k_unpalettize<FMT_FP16>, grid, dim3(256), idx, idx_bytes, n, bits, lut, out);
    return hipSuccess;
}

}  // namespace edkm
