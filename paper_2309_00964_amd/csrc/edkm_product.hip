// Products with an epilogue for gfx950 (MI355X): y = act(x W^T + bias) + residual with
// 16-bit weights, the products of its backward pass and the gradient at its activation.

#include "edkm_product.h"

#include <algorithm>

namespace edkm {

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

// Eight outputs from column c of row r on; a PLAIN epilogue only rounds and stores.
template <int F, bool PLAIN>
__device__ __forceinline__ void finish8(const ProductArgs& p, int r, int c, float (&z)[8]) {
    if (r >= p.rows || c >= p.cols) return;
    uint16_t* out = p.out + (int64_t)r * p.ldo + c;
    if (c + 8 <= p.cols) {
        s16x8 v;
        if (!PLAIN) {
            if (p.bias) {
                v = reinterpret_cast<const S16x8*>(p.bias + c)->v;
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] += to_f32<F>((uint16_t)v[q]);
            }
            if (p.z) {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = (short)keep_z<F>(z[q]);
                reinterpret_cast<S16x8*>(p.z + (int64_t)r * p.cols + c)->v = v;
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
                v = reinterpret_cast<const S16x8*>(p.res + (int64_t)r * p.ldr + c)->v;
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] += to_f32<F>((uint16_t)v[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = (short)to_16<F>(z[q]);
        reinterpret_cast<S16x8*>(out)->v = v;
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
#pragma unroll 4
    for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += *reinterpret_cast<const f32x4*>(at + s * stride + j * 256);
#pragma unroll
    for (int j = 0; j < 4; ++j) epi_put(lds, lane, j, acc[j]);
    epi_rows<F, PLAIN>(p, lds, lane, 1, r, c);
}

// ----------------------------------------------------------------------------
// the gradient at the activation

// A thread takes eight columns of every fourth row of the block's; one pass over dy and z
// (bound by its bytes: 6 B per element with an activation, 2 B without) writes dz and sums
// the bias gradient in fp32, unrounded.
template <int F, int ACT>
__global__ void __launch_bounds__(256) k_dz(DzArgs a) {
    __shared__ float red[4][DZ_COLS];
    const int lane = threadIdx.x & 63, q = threadIdx.x >> 6;
    // workgroups go column block by column block through a chunk of rows
    const uint32_t nc = (a.cols + DZ_COLS - 1) / DZ_COLS, cb = blockIdx.x % nc, chunk = blockIdx.x / nc;
    const int c = cb * DZ_COLS + lane * 8, left = a.cols - c;
    const int r0 = chunk * a.per, r1 = min(r0 + a.per, a.rows);
    float sum[8] = {};
    if (left > 0) {
#pragma unroll 2
        for (int r = r0 + q; r < r1; r += 4) {
            const s16x8 d = row8(a.dy + (int64_t)r * a.lddy + c, left);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = to_f32<F>((uint16_t)d[j]);
            if (ACT != ACT_NONE) {
                const s16x8 z = row8(a.z + (int64_t)r * a.cols + c, left);
                uint16_t* out = a.dz + (int64_t)r * a.lddz + c;
                s16x8 o;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] *= act_slope(to_f32<F>((uint16_t)z[j]), ACT);
                    o[j] = (short)to_16<F>(v[j]);
                }
                *reinterpret_cast<s16x8*>(out) = left >= 8 ? o : keep_first(o, left);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
    }
    if (!a.dbias) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) red[q][lane * 8 + j] = sum[j];
    __syncthreads();
    for (int i = threadIdx.x; i < DZ_COLS; i += 256)
        if (cb * DZ_COLS + i < (uint32_t)a.cols)
            a.part[(int64_t)chunk * a.cols + cb * DZ_COLS + i] = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
}

// 32 columns per workgroup, their chunks shared by 32 threads each
template <int F>
__global__ void __launch_bounds__(1024) k_dbias(DzArgs a, int chunks) {
    __shared__ float red[32][33];
    const int l = threadIdx.x & 31, q = threadIdx.x >> 5, c = blockIdx.x * 32 + l;
    float sum = 0.f;
    if (c < a.cols)
#pragma unroll 4
        for (int i = q; i < chunks; i += 32) sum += a.part[(int64_t)i * a.cols + c];
    red[q][l] = sum;
    __syncthreads();
    // column q's 32 sums lie in this half wave
    sum = red[l][q];
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor(sum, o, 32);
    const int mine = blockIdx.x * 32 + q;
    if (l == 0 && mine < a.cols) a.dbias[mine] = to_16<F>(sum);
}

// ----------------------------------------------------------------------------
// launches

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
    if (q.tile == 256) return tiled<F, OPA, OPB, 256, 2, 4, true>(p, q, s);
    return q.direct ? tiled<F, OPA, OPB, 128, 2, 2, true>(p, q, s) : tiled<F, OPA, OPB, 128, 2, 2, false>(p, q, s);
}

template <int F>
static hipError_t product_f(ProductArgs p, int opa, int opb, float* part, hipStream_t s) {
    if (opa == OP_ROWS && opb != OP_DEPTH && p.rows <= FEW) return launch_few(p, F, opb == OP_PALETTE ? p.bits : 0, s);
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

// A tile and a split of the depths.  What bounds a tile is bringing its operands into LDS,
// whose bytes per product fall with the tile's side, so the larger one where it gives most
// CUs a tile; two of the smaller share a CU, and its depths are split where they are few.
// Unaligned operands, whose way through registers the larger tile has no room for, take
// the smaller.
static void shape_plan(int64_t rows, int64_t cols, int64_t depth, bool direct, ProductPlan& q) {
    auto tiles = [&](int64_t b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
    const int64_t steps = std::max<int64_t>(1, (depth + 63) / 64);
    q.direct = direct;
    q.tile = direct && tiles(256) >= 192 ? 256 : 128;
    q.splits = 1;
    const int64_t t = tiles(q.tile);
    if (q.tile == 128 && t < 256) q.splits = (int)std::max<int64_t>(1, std::min<int64_t>({512 / t, steps / 4, 64}));
    q.split_steps = (int)((steps + q.splits - 1) / q.splits);
    q.splits = (int)((steps + q.split_steps - 1) / q.split_steps);
}

size_t product_part_bytes(int64_t rows, int64_t cols, int64_t depth) {
    size_t most = 0;
    for (const bool direct : {false, true}) {
        ProductPlan q{};
        shape_plan(rows, cols, depth, direct, q);
        if (q.splits > 1)
            most = std::max(most, (size_t)((rows + q.tile - 1) / q.tile) * ((cols + q.tile - 1) / q.tile) * q.tile * q.tile * 4 * q.splits);
    }
    return most;
}

ProductPlan product_plan(const ProductArgs& p, int opa, int opb) {
    ProductPlan q{};
    auto whole = [&](const void* m, int64_t ld, int op) {
        return ((uintptr_t)m & 15) == 0 && ld % 8 == 0 && ld <= (1 << 22) && (op == OP_DEPTH || p.depth % 8 == 0 || p.padded);
    };
    shape_plan(p.rows, p.cols, p.depth, whole(p.a, p.lda, opa) && whole(p.b, p.ldb, opb), q);
    return q;
}

template <int F>
static hipError_t dz_f(const DzArgs& a, hipStream_t s) {
    const int chunks = (a.rows + a.per - 1) / a.per;
    if (chunks > 0 && (a.dbias || a.act != ACT_NONE))
    {
        const dim3 grid((uint32_t)((a.cols + DZ_COLS - 1) / DZ_COLS) * chunks);
        if (a.act == ACT_NONE) EDKM_GO((k_dz<F, ACT_NONE>), grid, dim3(256), a);
        else if (a.act == ACT_RELU) EDKM_GO((k_dz<F, ACT_RELU>), grid, dim3(256), a);
        else if (a.act == ACT_GELU) EDKM_GO((k_dz<F, ACT_GELU>), grid, dim3(256), a);
        else EDKM_GO((k_dz<F, ACT_SILU>), grid, dim3(256), a);
    }
    if (a.dbias) EDKM_GO(k_dbias<F>, dim3((a.cols + 31) / 32), dim3(1024), a, chunks);
    return hipSuccess;
}

hipError_t launch_dz(const DzArgs& a, int fmt, hipStream_t s) {
    return fmt == FMT_BF16 ? dz_f<FMT_BF16>(a, s) : dz_f<FMT_FP16>(a, s);
}

}  // namespace edkm
