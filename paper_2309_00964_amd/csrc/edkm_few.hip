// Products of few tokens with 16-bit or palettized weights, and the 16-bit weights of a
// palette, for gfx950 (MI355X).

#include "edkm_product.h"

namespace edkm {

// Thirty-two weights per thread: 4 b bytes of indices, 64 bytes out, bound by the bytes
// written.  Unaligned or ragged ends take eight indices at a time, any alignment.
template <int F, int BITS>
__global__ void __launch_bounds__(256) k_unpalettize(const uint8_t* idx, uint64_t nbytes, uint64_t n, const float* lut,
                                                     uint16_t* out, int aligned) {
    Decoder<F> dec;
    dec.init(lut, BITS);
    // a wave's 2048 weights; its j-th store covers 512 consecutive ones, eight per lane
    const uint64_t base = ((uint64_t)blockIdx.x * 256 + (threadIdx.x & ~63)) * 32;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint64_t i = base + j * 512 + lane * 8;
        if (i >= n) return;
        const s16x8 v = dec.eight(load_idx8(idx, nbytes, i, BITS), BITS);
        if (aligned && i + 8 <= n) {
            *reinterpret_cast<s16x8*>(out + i) = v;
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (i + q < n) out[i + q] = (uint16_t)v[q];
        }
    }
}

// ----------------------------------------------------------------------------
// products of few tokens

// Table of pairs (4-bit palettes): entry e holds the values of indices e mod 2^b and e / 2^b, once per LDS
// bank, so that the lanes of a wave look up without conflicts.
constexpr int PAIR_BANKS = 32;

// A lane's weights of a run: 32 depths of each of its NT rows, as 16-bit values (BITS 0) or
// as packed indices.  WHOLE: 32 depths are 4 BITS bytes on a 4-byte boundary (16-bit
// values: on a 16-byte one), all there or none; else any alignment and end.
template <int F, int BITS, bool WHOLE>
struct FewWeights {
    uint32_t raw[BITS ? 4 : 1];
    s16x8 w[BITS ? 1 : 4];

    __device__ __forceinline__ void load(const ProductArgs& p, int row, int d) {
        const int left = p.depth - d;
        if constexpr (BITS == 0) {
            const uint16_t* at = p.b + (int64_t)row * p.ldb + d;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (WHOLE) w[j] = left > 0 ? *reinterpret_cast<const s16x8*>(at + j * 8) : s16x8{};
                else w[j] = row8(at + j * 8, left - j * 8);
            }
        } else if constexpr (WHOLE) {
            const uint32_t* at = reinterpret_cast<const uint32_t*>(p.idx) + ((uint64_t)row * (uint32_t)p.depth + d) / 32 * BITS;
#pragma unroll
            for (int j = 0; j < BITS; ++j) raw[j] = left > 0 ? at[j] : 0;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                raw[j] = left > j * 8 ? load_idx8(p.idx, p.idx_bytes, (uint64_t)row * (uint32_t)p.depth + d + j * 8, BITS) : 0;
        }
    }
    // the values of depths 8 j .. 8 j + 7: up to eight entries by lookups in registers,
    // sixteen from the table of pairs
    __device__ __forceinline__ s16x8 eight(const Decoder<F>& dec, const uint32_t* mine, int j, int left) const {
        if constexpr (BITS == 0) {
            return w[j];
        } else {
            typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
            uint32_t v;
            if (WHOLE) {
                constexpr int BPJ = 8 * BITS;                 // bits of eight indices
                const int at = j * BPJ, q = at / 32, sh = at % 32;
                v = sh + BPJ > 32 ? __builtin_amdgcn_alignbit(raw[q + 1 < 4 ? q + 1 : 3], raw[q], sh) : raw[q] >> sh;
            } else {
                v = raw[j];
            }
            s16x8 e;
            if constexpr (BITS < 4) {
                e = dec.eight(v, BITS);
            } else {
                u32x4 r;
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = mine[__builtin_amdgcn_ubfe(v, 2 * BITS * i, 2 * BITS) * PAIR_BANKS];
                e = __builtin_bit_cast(s16x8, r);
            }
            return WHOLE || left >= 8 ? e : keep_first(e, left);
        }
    }
};

// Up to 16 MT tokens against 16 NT weight rows per workgroup.  The waves share the depths by
// runs of 128 and add their sums through LDS.  The MFMA takes the weights as its rows: lane
// l holds row l mod 16, depths 32 (l / 16) + 8 j + 0 .. 7 of a run at its j-th step, so its
// share of a palette's run is 4 b consecutive bytes.  Bound by the weights' bytes and by the
// latency of one round: a wave asks for its weights of U runs, and for U more ahead, before
// it waits for anything, the table included.
//
// XL: the tokens (up to FEW_X bytes) wait in LDS.  Read from memory they are four times the
// bytes of a 4-bit palette, lane by lane, and each round waits for them.
constexpr int FEW_X = 48 * 1024;
__host__ __device__ constexpr int few_x_row(int depth) { return depth * 2 + 16; }   // bytes: rows fall on different banks

template <int F, int BITS, bool WHOLE, int MT, int NT, int U, int NW, bool XL>
__global__ void __launch_bounds__(NW * 64) k_few(ProductArgs p) {
    constexpr int ENTRIES = 1 << (2 * BITS);
    constexpr int TABLE = BITS == 4 ? ENTRIES * PAIR_BANKS : 0, SUMS = NW * MT * NT * 256, XW = XL ? FEW_X / 4 : 0;
    // the table and the tokens, and after the last of them the waves' sums
    __shared__ __attribute__((aligned(16))) uint32_t lds[TABLE + XW > SUMS ? TABLE + XW : SUMS];
    char* xl = reinterpret_cast<char*>(lds + TABLE);
    __shared__ uint16_t tab[KMAX];
    uint32_t* pairs = lds;
    float* red = reinterpret_cast<float*>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int l = lane & 15, g = lane >> 4;
    const int c0 = blockIdx.x * 16 * NT;
    const int runs = (p.depth + 127) / 128;
    FewWeights<F, BITS, WHOLE> now[U][NT], next[BITS ? U : 1][BITS ? NT : 1];
    s16x8 x[U][MT][4];
    int row[NT];
    auto load_x = [&](int t0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int d = (t0 + u * nw) * 128 + g * 32, left = p.depth - d;
            if constexpr (XL) {
                // lanes without a token repeat the first one's: their columns are not used
                const char* at = xl + (l < p.rows ? l : 0) * few_x_row(p.depth) + min(d, p.depth - 32) * 2;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[u][0][j] = *reinterpret_cast<const s16x8*>(at + j * 16);
                    if (left <= 0) x[u][0][j] = s16x8{};
                }
                continue;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                // lanes without a token load nothing: what a load costs here is its lanes, not its bytes
                const int r = i * 16 + l;
                const uint16_t* at = p.a + (int64_t)r * p.lda + d;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[u][i][j] = s16x8{};
                if (r < p.rows && left > 0)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (WHOLE) x[u][i][j] = *reinterpret_cast<const s16x8*>(at + j * 8);
                        else x[u][i][j] = row8(at + j * 8, left - j * 8);
                    }
            }
        }
    };
#pragma unroll
    for (int n = 0; n < NT; ++n) row[n] = min(c0 + n * 16 + l, p.cols - 1);
    auto load_w = [&](auto& to, int t0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n) to[u][n].load(p, row[n], (t0 + u * nw) * 128 + g * 32);
    };
    load_w(now, wave);
    if constexpr (XL) {
        const int pieces = p.depth / 8;
        for (int i = threadIdx.x; i < p.rows * pieces; i += blockDim.x) {
            const int r = i / pieces, q = i % pieces;
            *reinterpret_cast<s16x8*>(xl + r * few_x_row(p.depth) + q * 16) = *reinterpret_cast<const s16x8*>(p.a + (int64_t)r * p.lda + q * 8);
        }
        if (BITS != 4) __syncthreads();
    } else {
        load_x(wave);
    }
    Decoder<F> dec;
    if constexpr (BITS == 1 || BITS == 2 || BITS == 3) dec.init(p.lut, BITS);
    if constexpr (BITS == 4) {
        if (threadIdx.x < (1 << BITS)) tab[threadIdx.x] = to_16<F>(p.lut[threadIdx.x]);
        __syncthreads();
        for (int i = threadIdx.x; i < ENTRIES * PAIR_BANKS; i += blockDim.x) {
            const int e = i / PAIR_BANKS;
            pairs[i] = (uint32_t)tab[e & ((1 << BITS) - 1)] | ((uint32_t)tab[e >> BITS] << 16);
        }
        __syncthreads();
    }
    if constexpr (XL) load_x(wave);
    const uint32_t* mine = pairs + (lane & (PAIR_BANKS - 1));
    f32x4 acc[MT][NT] = {};
    for (int t = wave; t < runs; t += nw * U) {
        if constexpr (BITS != 0) load_w(next, t + nw * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int left = p.depth - ((t + u * nw) * 128 + g * 32);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    s16x8 w = now[u][n].eight(dec, mine, j, left - j * 8);
                    if (BITS && WHOLE && left <= 0) w = s16x8{};
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i][n] = mfma16<F>(w, x[u][i][j], acc[i][n]);
                }
        }
        if (t + nw * U < runs) {
            load_x(t + nw * U);
            if constexpr (BITS != 0) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int n = 0; n < NT; ++n) now[u][n] = next[u][n];
            } else {
                load_w(now, t + nw * U);
            }
        }
    }
    if (BITS == 4 || XL) __syncthreads();
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
            *reinterpret_cast<f32x4*>(red + (((wave * MT + i) * NT + n) * 64 + lane) * 4) = acc[i][n];
    __syncthreads();
    for (int e = threadIdx.x; e < min(p.rows, 16 * MT) * NT * 16; e += blockDim.x) {
        const int n = e % (16 * NT), r = e / (16 * NT), i = r >> 4;
        const int at = ((i * NT + (n >> 4)) * 64 + ((n & 15) >> 2) * 16 + (r & 15)) * 4 + (n & 3);
        float z = 0.f;
        for (int w = 0; w < nw; ++w) z += red[w * MT * NT * 256 + at];
        const int col = c0 + n;
        if (col >= p.cols) continue;
        if (p.bias) z += to_f32<F>(p.bias[col]);
        if (p.z) p.z[(int64_t)r * p.cols + col] = keep_z<F>(z);
        float y = act_value(z, p.act);
        if (p.res) y += to_f32<F>(p.res[(int64_t)r * p.ldr + col]);
        p.out[(int64_t)r * p.ldo + col] = to_16<F>(y);
    }
}

template <int F, int BITS, bool WHOLE, int MT, int NT, int U, int NW, bool XL>
static hipError_t few_go(const ProductArgs& p, hipStream_t s) {
    const int runs = (p.depth + 127) / 128;
    int nw = 1;
    while (nw < runs && nw < NW) nw *= 2;
    EDKM_GO((k_few<F, BITS, WHOLE, MT, NT, U, NW, XL>), dim3((uint32_t)(((int64_t)p.cols + 16 * NT - 1) / (16 * NT))), dim3(nw * 64), p);
    return hipSuccess;
}

template <int F, int BITS, bool WHOLE>
static hipError_t few_bits(const ProductArgs& p, hipStream_t s) {
    const int64_t tiles = ((int64_t)p.cols + 15) / 16;
    if constexpr (!WHOLE) {
        if (p.rows <= 16) return few_go<F, BITS, WHOLE, 1, 1, 1, 16, false>(p, s);
        return p.rows <= 32 ? few_go<F, BITS, WHOLE, 2, 1, 1, 8, false>(p, s) : few_go<F, BITS, WHOLE, 4, 1, 1, 8, false>(p, s);
    } else {
        constexpr int U1 = BITS ? 3 : 1, U2 = BITS ? 2 : 1;
        const bool xl = BITS && (int64_t)p.rows * few_x_row(p.depth) <= FEW_X;
        if (p.rows <= 16) {
            if (tiles <= 256) return xl ? few_go<F, BITS, WHOLE, 1, 1, U1, 16, BITS != 0>(p, s) : few_go<F, BITS, WHOLE, 1, 1, U2, 16, false>(p, s);
            if (tiles <= 512 || !BITS) return xl ? few_go<F, BITS, WHOLE, 1, 2, U2, 16, BITS != 0>(p, s) : few_go<F, BITS, WHOLE, 1, 2, U2, 16, false>(p, s);
            return xl ? few_go<F, BITS, WHOLE, 1, 3, U2, 16, BITS != 0>(p, s) : few_go<F, BITS, WHOLE, 1, 3, U2, 16, false>(p, s);
        }
        if (p.rows <= 32) {
            if (tiles <= 256) return few_go<F, BITS, WHOLE, 2, 1, 1, 8, false>(p, s);
            return tiles <= 512 ? few_go<F, BITS, WHOLE, 2, 2, 1, 8, false>(p, s) : few_go<F, BITS, WHOLE, 2, 3, 1, 8, false>(p, s);
        }
        if (tiles <= 256) return few_go<F, BITS, WHOLE, 4, 1, 1, 8, false>(p, s);
        return tiles <= 512 ? few_go<F, BITS, WHOLE, 4, 2, 1, 8, false>(p, s) : few_go<F, BITS, WHOLE, 4, 3, 1, 8, false>(p, s);
    }
}

template <int F>
static hipError_t few(const ProductArgs& p, int bits, hipStream_t s) {
    const bool x16 = ((uintptr_t)p.a & 15) == 0 && p.lda % 8 == 0 && p.depth % 32 == 0;
    const bool whole = x16 && (bits ? ((uintptr_t)p.idx & 3) == 0 : ((uintptr_t)p.b & 15) == 0 && p.ldb % 8 == 0);
    switch (bits) {
    case 1: return whole ? few_bits<F, 1, true>(p, s) : few_bits<F, 1, false>(p, s);
    case 2: return whole ? few_bits<F, 2, true>(p, s) : few_bits<F, 2, false>(p, s);
    case 3: return whole ? few_bits<F, 3, true>(p, s) : few_bits<F, 3, false>(p, s);
    case 4: return whole ? few_bits<F, 4, true>(p, s) : few_bits<F, 4, false>(p, s);
    default: return whole ? few_bits<F, 0, true>(p, s) : few_bits<F, 0, false>(p, s);
    }
}

hipError_t launch_few(const ProductArgs& p, int fmt, int bits, hipStream_t s) {
    return fmt == FMT_BF16 ? few<FMT_BF16>(p, bits, s) : few<FMT_FP16>(p, bits, s);
}

template <int F>
static hipError_t unpalettize_f(const uint8_t* idx, uint64_t nb, uint64_t n, int bits, const float* lut, uint16_t* out,
                                hipStream_t s) {
    const dim3 grid((uint32_t)((n + 8191) / 8192));
    const int al = ((uintptr_t)out & 15) == 0;
    if (bits == 1) EDKM_GO((k_unpalettize<F, 1>), grid, dim3(256), idx, nb, n, lut, out, al);
    else if (bits == 2) EDKM_GO((k_unpalettize<F, 2>), grid, dim3(256), idx, nb, n, lut, out, al);
    else if (bits == 3) EDKM_GO((k_unpalettize<F, 3>), grid, dim3(256), idx, nb, n, lut, out, al);
    else EDKM_GO((k_unpalettize<F, 4>), grid, dim3(256), idx, nb, n, lut, out, al);
    return hipSuccess;
}

hipError_t launch_unpalettize(const uint8_t* idx, uint64_t idx_bytes, uint64_t n, int bits, int fmt, const float* lut,
                              uint16_t* out, hipStream_t s) {
    return fmt == FMT_BF16 ? unpalettize_f<FMT_BF16>(idx, idx_bytes, n, bits, lut, out, s)
                           : unpalettize_f<FMT_FP16>(idx, idx_bytes, n, bits, lut, out, s);
}

}  // namespace edkm
