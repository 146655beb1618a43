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

template <int F>
static hipError_t product_f(ProductArgs p, int opa, int opb, float* part, hipStream_t s) {
    if (opb == OP_PALETTE) {
        const dim3 grid((p.cols + TN - 1) / TN, (p.rows + TM - 1) / TM);
        EDKM_GO((k_product<F, OP_ROWS, OP_PALETTE>), grid, dim3(256), p);
        return hipSuccess;
    }
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

hipError_t launch_unpalettize(const uint8_t* idx, uint64_t idx_bytes, uint64_t n, int bits, int fmt, const float* lut,
                              uint16_t* out, hipStream_t s) {
    const dim3 grid((uint32_t)((n + 2047) / 2048));
    if (fmt == FMT_BF16) EDKM_GO(k_unpalettize<FMT_BF16>, grid, dim3(256), idx, idx_bytes, n, bits, lut, out);
    else EDKM_GO(k_unpalettize<FMT_FP16>, grid, dim3(256), idx, idx_bytes, n, bits, lut, out);
    return hipSuccess;
}

}  // namespace edkm
