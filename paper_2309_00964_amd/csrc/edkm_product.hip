// Products with an epilogue for gfx950 (MI355X): y = act(x W^T + bias) + residual with
// 16-bit or palettized weights, the products of its backward pass, and the 16-bit
// weights of a palette.

#include "edkm_layer.h"

#include <hip/hip_fp16.h>
#include <algorithm>

namespace edkm {

typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
struct __attribute__((packed)) S16x8 { s16x8 v; };

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
__device__ __forceinline__ s16x8 row8(const uint16_t* q, int left) {
    if (left >= 8) return reinterpret_cast<const S16x8*>(q)->v;
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
// tiled products

// One operand's tile of R output indices x 64 depths in LDS, filled by 16-byte pieces.
//
// OP_ROWS: [R][64], a row is 128 bytes; piece c of row r lies at place c ^ (r & 7), so
// that the 16-byte fragment reads of sixteen rows fall on different banks.
// OP_DEPTH: [64][R]; fragments are read transposed (ds_read_b64_tr_b16: sixteen lanes
// read 4 depths x 16 indices and each gets the 4 depths of its index).  The 32-byte
// units of depth d are permuted by an exclusive or with (d & 3) + 4 (d >> 3 & 3), since
// one read takes 16 depths of the same unit.
template <int OP, int R, int NW>
struct Tile {
    static constexpr int BYTES = R * 128;
    static constexpr int PER = BYTES / 1024 / NW;     // pieces of 1 KiB per wave
    static constexpr int LPD = R / 8;                 // OP_DEPTH: lanes (pieces) per depth
    static constexpr int UM = R / 16 - 1;             // OP_DEPTH: mask of the units

    __device__ __forceinline__ static int swz(int d) { return ((d & 3) | ((d >> 1) & 12)) & UM; }
    // place of lane's piece i of wave w: (index or first index, depth) of its 8 elements
    __device__ __forceinline__ static void place(int w, int i, int lane, int& idx, int& d) {
        const int q = w * PER + i;
        if (OP == OP_DEPTH) {
            d = q * (64 / LPD) + lane / LPD;
            const int p = lane % LPD;
            idx = (((p >> 1) ^ swz(d)) * 2 + (p & 1)) * 8;
        } else {
            idx = q * 8 + (lane >> 3);
            d = ((lane & 7) ^ (lane >> 3)) * 8;
        }
    }
    // fragment reads: index base u0 (multiple of 16 times the wave's tiles)
    int off[2];
    __device__ __forceinline__ void init(int base, int lane) {
        const int l = lane & 15, g = lane >> 4;
        if (OP == OP_DEPTH) {
            const int d = g * 8 + (l >> 2);
            off[0] = d * (R * 2) + (((base >> 4) ^ swz(d)) * 32) + (l & 3) * 8;
            off[1] = 0;
        } else {
            off[0] = (base + l) * 128 + ((g ^ (l & 7)) * 16);
            off[1] = (base + l) * 128 + (((g + 4) ^ (l & 7)) * 16);
        }
    }
    __device__ __forceinline__ s16x8 frag(const char* lds, int t, int ks) const {
        if constexpr (OP == OP_DEPTH) {
            typedef __attribute__((address_space(3))) s16x4 lds4;
            const char* p = lds + (off[0] ^ (t * 32)) + ks * (R * 64);
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)p);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p + R * 8));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            return *reinterpret_cast<const s16x8*>(lds + off[ks] + t * 2048);
        }
    }
};

// A buffer's bytes from `p` on that a tile may read: range-checked, zeros past the end.
constexpr int OUT_OF_RANGE = 0x7FFFFFF0;
typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ __forceinline__ rsrc_t buffer_at(const void* p, int64_t bytes) {
    const int n = bytes < 0 ? 0 : bytes > OUT_OF_RANGE ? OUT_OF_RANGE : (int)((bytes + 3) & ~3ll);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, n, 0x00027000);
}

// Brings an operand's tiles into LDS.  DIRECT: by buffer loads that write LDS, for rows of
// memory that start on 16 bytes (and whole pieces of 8 depths for OP_ROWS); else through
// registers, by loads of any alignment.
template <int OP, int R, int NW, bool DIRECT>
struct Feed {
    typedef Tile<OP, R, NW> T;
    const uint16_t* m;       // the tile's first element at depth 0
    int64_t ld;
    int limit, depth;        // output indices from m on; depths in all
    int wave, lane;
    int voff[T::PER], vd[T::PER];
    s16x8 reg[DIRECT ? 1 : T::PER];

    __device__ __forceinline__ void init(const uint16_t* base, int64_t ld_, int first, int count, int depth_, int wave_,
                                         int lane_) {
        ld = ld_;
        m = OP == OP_DEPTH ? base + first : base + (int64_t)first * ld;
        limit = count - first;
        depth = depth_;
        wave = wave_;
        lane = lane_;
#pragma unroll
        for (int i = 0; i < T::PER; ++i) {
            int idx, d;
            T::place(wave, i, lane, idx, d);
            vd[i] = d;
            voff[i] = OP == OP_DEPTH ? (int)((d * ld + idx) * 2) : (int)((idx * ld + d) * 2);
        }
    }
    // start bringing in depths d0 .. d0 + 63
    __device__ __forceinline__ void start(char* lds, int d0) {
        if constexpr (DIRECT) {
            rsrc_t r;
            if (OP == OP_DEPTH)
                r = buffer_at(m + (int64_t)d0 * ld, ((int64_t)(depth - 1 - d0) * ld + limit) * 2);
            else
                r = buffer_at(m + d0, ((int64_t)(limit - 1) * ld + depth - d0) * 2);
            const bool tail = OP != OP_DEPTH && d0 + 64 > depth;
#pragma unroll
            for (int i = 0; i < T::PER; ++i) {
                const int off = tail && d0 + vd[i] >= depth ? OUT_OF_RANGE : voff[i];
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    r, (__attribute__((address_space(3))) void*)(lds + (wave * T::PER + i) * 1024), 16, off, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < T::PER; ++i) {
                int idx, d;
                T::place(wave, i, lane, idx, d);
                reg[i] = fetch(idx, d0 + d);
            }
        }
    }
    // what start() left in registers
    __device__ __forceinline__ void finish(char* lds) {
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < T::PER; ++i)
                *reinterpret_cast<s16x8*>(lds + (wave * T::PER + i) * 1024 + lane * 16) = reg[i];
    }
    __device__ __forceinline__ s16x8 fetch(int idx, int d) const {
        s16x8 v = {};
        if (OP == OP_DEPTH) {
            if (d >= depth || idx >= limit) return v;
            const uint16_t* q = m + (int64_t)d * ld + idx;
            if (idx + 8 <= limit) return reinterpret_cast<const S16x8*>(q)->v;
            for (int j = 0; j < 8; ++j)
                if (idx + j < limit) v[j] = (short)q[j];
        } else {
            if (idx >= limit || d >= depth) return v;
            const uint16_t* q = m + (int64_t)idx * ld + d;
            if (d + 8 <= depth) return reinterpret_cast<const S16x8*>(q)->v;
            for (int j = 0; j < 8; ++j)
                if (d + j < depth) v[j] = (short)q[j];
        }
        return v;
    }
};

// Tile (x, y) of workgroup w: each of the eight XCDs (workgroups go to them in turn) takes
// a run of tiles, and within a run eight tile rows are walked column by column, so that
// the XCD's L2 holds the operands that its tiles share.
__device__ __forceinline__ void tile_of(uint32_t w, uint32_t nx, uint32_t ny, uint32_t& x, uint32_t& y) {
    const uint32_t total = nx * ny, per = total / 8, more = total % 8;
    const uint32_t xcd = w % 8, t = xcd * per + min(xcd, more) + w / 8;
    const uint32_t group = t / (8 * nx), first = group * 8, h = min(8u, ny - first);
    const uint32_t in = t - group * 8 * nx;
    y = first + in % h;
    x = in / h;
}

// ----------------------------------------------------------------------------
// epilogue

struct __attribute__((packed)) U16x8 { s16x8 v; };

// Eight outputs from column c of row r on; a PLAIN epilogue only rounds and stores.
template <int F, bool PLAIN>
__device__ __forceinline__ void finish8(const ProductArgs& p, int r, int c, float (&z)[8]) {
    if (r >= p.rows || c >= p.cols) return;
    uint16_t* out = p.out + (int64_t)r * p.ldo + c;
    if (c + 8 <= p.cols) {
        s16x8 v;
        if (!PLAIN) {
            if (p.bias) {
                v = reinterpret_cast<const U16x8*>(p.bias + c)->v;
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] += to_f32<F>((uint16_t)v[q]);
            }
            if (p.z) {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = (short)keep_z<F>(z[q]);
                reinterpret_cast<U16x8*>(p.z + (int64_t)r * p.cols + c)->v = v;
            }
            if (p.act == ACT_RELU) {
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] = act_value(z[q], ACT_RELU);
            } else if (p.act == ACT_GELU) {
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] = act_value(z[q], ACT_GELU);
            } else if (p.act == ACT_SILU) {
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] = act_value(z[q], ACT_SILU);
            }
            if (p.res) {
                v = reinterpret_cast<const U16x8*>(p.res + (int64_t)r * p.ldr + c)->v;
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] += to_f32<F>((uint16_t)v[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = (short)to_16<F>(z[q]);
        reinterpret_cast<U16x8*>(out)->v = v;
        return;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if (c + q >= p.cols) break;
        float v = z[q];
        if (!PLAIN) {
            if (p.bias) v += to_f32<F>(p.bias[c + q]);
            if (p.z) p.z[(int64_t)r * p.cols + c + q] = keep_z<F>(v);
            v = act_value(v, p.act);
            if (p.res) v += to_f32<F>(p.res[(int64_t)r * p.ldr + c + q]);
        }
        out[q] = to_16<F>(v);
    }
}

// A wave's 16 x 64 block of sums as the MFMA leaves it (row lane & 15, four columns per
// tile of 16) goes through LDS, so that lanes take eight columns of a row: whole 128-byte
// lines to and from memory.  Its 16-byte places are permuted by the row.
constexpr int EPI_BYTES = 16 * 64 * 4;
__device__ __forceinline__ void epi_put(char* lds, int lane, int j, f32x4 v) {
    const int r = lane & 15;
    *reinterpret_cast<f32x4*>(lds + r * 256 + (((j * 4 + (lane >> 4)) ^ r) * 16)) = v;
}
template <int F, bool PLAIN>
__device__ __forceinline__ void epi_rows(const ProductArgs& p, const char* lds, int lane, int blocks, int r0, int c0) {
#pragma unroll 1
    for (int i = 0; i < blocks * 2; ++i) {
        const int r = i * 8 + (lane >> 3), q = (lane & 7) * 2, m = r & 15;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(lds + r * 256 + ((q ^ m) * 16));
        const f32x4 hi = *reinterpret_cast<const f32x4*>(lds + r * 256 + (((q + 1) ^ m) * 16));
        float z[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        finish8<F, PLAIN>(p, r0 + r, c0 + (lane & 7) * 8, z);
    }
}

// BM x BN outputs per workgroup, 64 depths a step in two LDS buffers; WM x WN waves.
// The sixteen-wide MFMA takes b's tile as its rows, so a lane ends with four consecutive
// columns of one output row.
template <int F, int OPA, int OPB, int BM, int BN, int WM, int WN, bool DIRECT>
__global__ void __launch_bounds__(WM * WN * 64, 2) k_tiled(ProductArgs p) {
    constexpr int NW = WM * WN, TR = BM / WM / 16, TC = BN / WN / 16;
    static_assert(TC == 4 && TR % 4 == 0, "a wave's columns are those of the epilogue");
    typedef Feed<OPA, BM, NW, DIRECT> FA;
    typedef Feed<OPB, BN, NW, DIRECT> FB;
    // four arrays, so that the compiler knows the loads of one buffer apart from the reads of the other
    __shared__ __attribute__((aligned(1024))) char a0[FA::T::BYTES], a1[FA::T::BYTES], b0[FB::T::BYTES], b1[FB::T::BYTES];
    static_assert(NW * 2 * EPI_BYTES <= FA::T::BYTES + FB::T::BYTES, "the epilogue's blocks fit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tx, ty;
    const uint32_t nx = (p.cols + BN - 1) / BN, ny = (p.rows + BM - 1) / BM;
    const uint32_t split = blockIdx.x / (nx * ny);
    tile_of(blockIdx.x % (nx * ny), nx, ny, tx, ty);
    const int r0 = ty * BM, c0 = tx * BN;
    const int wr = (wave / WN) * (BM / WM), wc = (wave % WN) * (BN / WN);
    FA fa;
    FB fb;
    fa.init(p.a, p.lda, r0, p.rows, p.depth, wave, lane);
    fb.init(p.b, p.ldb, c0, p.cols, p.depth, wave, lane);
    typename FA::T ta;
    typename FB::T tb;
    ta.init(wr, lane);
    tb.init(wc, lane);
    f32x4 acc[TR][TC] = {};
    const int first = split * p.split_steps, steps = min(first + p.split_steps, (p.depth + 63) / 64);

    auto step = [&](const char* a, const char* b, char* an, char* bn, int s) {
        if (s + 1 < steps) {
            fa.start(an, (s + 1) * 64);
            fb.start(bn, (s + 1) * 64);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            s16x8 va[TR], vb[TC];
#pragma unroll
            for (int j = 0; j < TC; ++j) vb[j] = tb.frag(b, j, ks);
#pragma unroll
            for (int i = 0; i < TR; ++i) va[i] = ta.frag(a, i, ks);
#pragma unroll
            for (int i = 0; i < TR; ++i)
#pragma unroll
                for (int j = 0; j < TC; ++j) acc[i][j] = mfma16<F>(vb[j], va[i], acc[i][j]);
        }
        if (s + 1 < steps) {
            fa.finish(an);
            fb.finish(bn);
        }
        __syncthreads();
    };
    if (first < steps) {
        fa.start(a0, first * 64);
        fb.start(b0, first * 64);
        fa.finish(a0);
        fb.finish(b0);
    }
    __syncthreads();
    for (int s = first; s < steps; s += 2) {
        step(a0, b0, a1, b1, s);
        if (s + 1 < steps) step(a1, b1, a0, b0, s + 1);
    }
    if (p.part) {
        float* at = p.part + ((int64_t)blockIdx.x * NW + wave) * (TR * 1024) + lane * 4;
#pragma unroll
        for (int i = 0; i < TR; ++i)
#pragma unroll
            for (int j = 0; j < TC; ++j) *reinterpret_cast<f32x4*>(at + (i * TC + j) * 256) = acc[i][j];
        return;
    }
    // each wave has two blocks of LDS: in a0/a1 the first half of the waves, in b0/b1 the others
    char* mine = (wave < NW / 2 ? a0 : b0) + (wave % (NW / 2)) * 2 * EPI_BYTES;
    static_assert(NW / 2 * 2 * EPI_BYTES <= (FA::T::BYTES < FB::T::BYTES ? FA::T::BYTES : FB::T::BYTES), "");
#pragma unroll
    for (int i = 0; i < TR; i += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < TC; ++j) epi_put(mine + h * EPI_BYTES, lane, j, acc[i + h][j]);
        epi_rows<F, OPB == OP_DEPTH>(p, mine, lane, 2, r0 + wr + i * 16, c0 + wc);
    }
}

// Adds the partial sums of a split product, split after split, and finishes them: one wave
// for 16 x 64 outputs.
template <int F, int BM, int BN, int WM, int WN, bool PLAIN>
__global__ void __launch_bounds__(64) k_join(ProductArgs p, int splits) {
    constexpr int NW = WM * WN, TR = BM / WM / 16;
    __shared__ __attribute__((aligned(16))) char lds[EPI_BYTES];
    const uint32_t nx = (p.cols + BN - 1) / BN, ny = (p.rows + BM - 1) / BM;
    const uint32_t w = blockIdx.x / (NW * TR);
    const int wave = blockIdx.x / TR % NW, i = blockIdx.x % TR, lane = threadIdx.x;
    uint32_t tx, ty;
    tile_of(w, nx, ny, tx, ty);
    const int r = ty * BM + wave / WN * (BM / WM) + i * 16, c = tx * BN + wave % WN * 64;
    if (r >= p.rows || c >= p.cols) return;
    f32x4 acc[4] = {};
    const float* at = p.part + ((int64_t)w * NW + wave) * (TR * 1024) + i * 1024 + lane * 4;
    const int64_t stride = (int64_t)nx * ny * NW * (TR * 1024);
    for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += *reinterpret_cast<const f32x4*>(at + s * stride + j * 256);
#pragma unroll
    for (int j = 0; j < 4; ++j) epi_put(lds, lane, j, acc[j]);
    epi_rows<F, PLAIN>(p, lds, lane, 1, r, c);
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
template <int F, int BITS, bool WHOLE, int MT, int NT, int U>
__global__ void __launch_bounds__(1024) k_few(ProductArgs p) {
    constexpr int ENTRIES = 1 << (2 * BITS);
    constexpr int TABLE = BITS == 4 ? ENTRIES * PAIR_BANKS : 0, SUMS = 16 * MT * NT * 256;
    // the table, and after the last lookup the waves' sums
    __shared__ __attribute__((aligned(16))) uint32_t lds[TABLE > SUMS ? TABLE : SUMS];
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
    load_x(wave);
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
    if (BITS == 4) __syncthreads();
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

template <int F, int OPA, int OPB, int B, int WM, int WN, bool DIRECT>
static hipError_t tiled(const ProductArgs& p, const ProductPlan& q, hipStream_t s) {
    const int64_t tiles = ((int64_t)p.cols + B - 1) / B * (((int64_t)p.rows + B - 1) / B);
    EDKM_GO((k_tiled<F, OPA, OPB, B, B, WM, WN, DIRECT>), dim3((uint32_t)(tiles * q.splits)), dim3(WM * WN * 64), p);
    if (q.splits > 1)
        EDKM_GO((k_join<F, B, B, WM, WN, OPB == OP_DEPTH>), dim3((uint32_t)(tiles * WM * WN * (B / WM / 16))), dim3(64), p, q.splits);
    return hipSuccess;
}

template <int F, int OPA, int OPB>
static hipError_t product_ab(const ProductArgs& p, const ProductPlan& q, hipStream_t s) {
    if (q.tile == 256)
        return q.direct ? tiled<F, OPA, OPB, 256, 2, 4, true>(p, q, s) : tiled<F, OPA, OPB, 256, 2, 4, false>(p, q, s);
    return q.direct ? tiled<F, OPA, OPB, 128, 2, 2, true>(p, q, s) : tiled<F, OPA, OPB, 128, 2, 2, false>(p, q, s);
}

template <int F, int BITS, bool WHOLE, int MT, int NT>
static hipError_t few_go(const ProductArgs& p, hipStream_t s) {
    constexpr int U = WHOLE && BITS && MT == 1 ? 2 : 1;
    const int runs = (p.depth + 127) / 128;
    int nw = 1;
    while (nw < runs && nw < 16) nw *= 2;
    EDKM_GO((k_few<F, BITS, WHOLE, MT, NT, U>), dim3((uint32_t)(((int64_t)p.cols + 16 * NT - 1) / (16 * NT))), dim3(nw * 64), p);
    return hipSuccess;
}

template <int F, int BITS, bool WHOLE>
static hipError_t few_bits(const ProductArgs& p, hipStream_t s) {
    const int64_t tiles = ((int64_t)p.cols + 15) / 16;
    if (!WHOLE) {
        if (p.rows <= 16) return few_go<F, BITS, WHOLE, 1, 1>(p, s);
        return p.rows <= 32 ? few_go<F, BITS, WHOLE, 2, 1>(p, s) : few_go<F, BITS, WHOLE, 4, 1>(p, s);
    }
    if (p.rows <= 16) {
        if (tiles <= 256) return few_go<F, BITS, WHOLE, 1, 1>(p, s);
        return tiles <= 512 || !BITS ? few_go<F, BITS, WHOLE, 1, 2>(p, s) : few_go<F, BITS, WHOLE, 1, 3>(p, s);
    }
    const bool wide = tiles >= 512;
    if (p.rows <= 32) return wide ? few_go<F, BITS, WHOLE, 2, 2>(p, s) : few_go<F, BITS, WHOLE, 2, 1>(p, s);
    return few_go<F, BITS, WHOLE, 4, 1>(p, s);
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

template <int F>
static hipError_t product_f(ProductArgs p, int opa, int opb, float* part, hipStream_t s) {
    if (opa == OP_ROWS && opb != OP_DEPTH && p.rows <= FEW) return few<F>(p, opb == OP_PALETTE ? p.bits : 0, s);
    const ProductPlan q = product_plan(p, opa, opb);
    p.split_steps = q.split_steps;
    p.part = q.splits > 1 ? part : nullptr;
    if (opa == OP_DEPTH) return product_ab<F, OP_DEPTH, OP_DEPTH>(p, q, s);
    if (opb == OP_DEPTH) return product_ab<F, OP_ROWS, OP_DEPTH>(p, q, s);
    return product_ab<F, OP_ROWS, OP_ROWS>(p, q, s);
}

hipError_t launch_product(const ProductArgs& p, int fmt, int opa, int opb, float* part, hipStream_t s) {
    return fmt == FMT_BF16 ? product_f<FMT_BF16>(p, opa, opb, part, s) : product_f<FMT_FP16>(p, opa, opb, part, s);
}

// A tile and a split of the depths from the sizes alone, so that a workspace can be sized
// before the call.
static void shape_plan(int64_t rows, int64_t cols, int64_t depth, ProductPlan& q) {
    auto tiles = [&](int64_t b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
    const int64_t steps = std::max<int64_t>(1, (depth + 63) / 64);
    q.tile = tiles(256) >= 192 ? 256 : 128;
    q.splits = 1;
    const int64_t t = tiles(q.tile);
    if (q.tile == 128 && t < 256) q.splits = (int)std::max<int64_t>(1, std::min<int64_t>({512 / t, steps / 4, 64}));
    q.split_steps = (int)((steps + q.splits - 1) / q.splits);
    q.splits = (int)((steps + q.split_steps - 1) / q.split_steps);
}

size_t product_part_bytes(int64_t rows, int64_t cols, int64_t depth) {
    ProductPlan q{};
    shape_plan(rows, cols, depth, q);
    if (q.splits <= 1) return 0;
    return (size_t)((rows + q.tile - 1) / q.tile) * ((cols + q.tile - 1) / q.tile) * q.tile * q.tile * 4 * q.splits;
}

ProductPlan product_plan(const ProductArgs& p, int opa, int opb) {
    ProductPlan q{};
    shape_plan(p.rows, p.cols, p.depth, q);
    auto whole = [&](const void* m, int64_t ld, int op) {
        return ((uintptr_t)m & 15) == 0 && ld % 8 == 0 && ld <= (1 << 22) && (op == OP_DEPTH || p.depth % 8 == 0);
    };
    q.direct = whole(p.a, p.lda, opa) && whole(p.b, p.ldb, opb);
    return q;
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
