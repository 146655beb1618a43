// The tiled product kernels, for 16-bit and for palettized weights.
#pragma once
#include "edkm_product.h"

#include <type_traits>

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
    __device__ __forceinline__ void finish(char* lds, int) {
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

// A palette's tile, as an OP_ROWS one: every piece is the B bytes of eight indices, looked up
// by pairs.  The bytes of a step are read one step before they are looked up, and the values
// go to LDS between a step's two halves, so that the lookups run under the matrix
// instructions (written at the step's end the product took 24.2 -> 25.5 us for 256 tokens of
// 4096 x 4096).  For rows of whole pieces and palettes of four bytes at least (the last
// bytes are read by a load that ends with them).
template <int F, int B, int R, int NW>
struct PaletteFeed {
    typedef Tile<OP_ROWS, R, NW> T;
    static constexpr int COPIES = B == 4 ? 16 : PAIR_BANKS;      // of the table's entries: two workgroups have 160 KiB
    static constexpr int TABLE = (1 << (2 * B)) * COPIES;        // 32-bit words
    const uint8_t* at;       // the tile's first row
    const char* mine;        // the lane's copy of the table
    uint32_t last;           // where the last load may start
    int depth, wave, lane;
    uint32_t voff[T::PER];
    int vd[T::PER];
    uint32_t raw[T::PER], back[T::PER];
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    u32x4 val[T::PER];

    __device__ __forceinline__ void init(const ProductArgs& p, uint32_t* table, int first, int wave_, int lane_) {
        const uint64_t row_bytes = (uint64_t)p.depth / 8 * B;
        at = p.idx + first * row_bytes;
        last = (uint32_t)min(p.idx_bytes - first * row_bytes - 4, (uint64_t)0x7FFFFFFF);
        if (p.idx_bytes < first * row_bytes + 4) {     // the last row's few bytes: one row of less than four
            at = p.idx + (p.idx_bytes - 4);
            last = 0;
        }
        depth = p.depth;
        wave = wave_;
        lane = lane_;
        mine = reinterpret_cast<const char*>(table + (lane & (COPIES - 1)));
        const uint32_t skip = (uint32_t)(p.idx + first * row_bytes - at);
#pragma unroll
        for (int i = 0; i < T::PER; ++i) {
            int idx, d;
            T::place(wave, i, lane, idx, d);
            vd[i] = d;
            voff[i] = skip + (uint32_t)min(idx, p.cols - 1 - first) * (uint32_t)row_bytes + d / 8 * B;
        }
    }
    static __device__ __forceinline__ void fill(uint32_t* table, const float* lut) {
        for (int i = threadIdx.x; i < TABLE; i += NW * 64) {
            const int e = i / COPIES;
            table[i] = (uint32_t)to_16<F>(lut[e & ((1 << B) - 1)]) | ((uint32_t)to_16<F>(lut[e >> B]) << 16);
        }
    }
    // reads the bytes of depths d0 .. d0 + 63
    __device__ __forceinline__ void load(int d0) {
#pragma unroll
        for (int i = 0; i < T::PER; ++i) {
            const uint32_t want = voff[i] + (uint32_t)(d0 / 8) * B, o = min(want, last);
            back[i] = (want - o) * 8;
            raw[i] = reinterpret_cast<const U32*>(at + o)->v;
        }
    }
    // looks up depths d0 .. d0 + 63, whose bytes are there, and reads the next ones'
    __device__ __forceinline__ void start(char*, int d0) {
        constexpr uint32_t MASK = ((1u << (2 * B)) - 1) * (COPIES * 4);
        constexpr int UP = COPIES == 16 ? 6 : 7;
#pragma unroll
        for (int i = 0; i < T::PER; ++i) {
            const uint32_t v = raw[i] >> (back[i] & 31);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int sh = 2 * B * j - UP;
                const uint32_t e = (sh < 0 ? v << (sh < 0 ? -sh : 0) : v >> (sh < 0 ? 0 : sh)) & MASK;
                val[i][j] = *reinterpret_cast<const uint32_t*>(mine + e);
            }
        }
        load(d0 + 64);
    }
    __device__ __forceinline__ void finish(char* lds, int d0) {
#pragma unroll
        for (int i = 0; i < T::PER; ++i) {
            u32x4 w = val[i];
            if (d0 + 64 > depth && d0 + vd[i] >= depth) w = u32x4{};
            *reinterpret_cast<u32x4*>(lds + (wave * T::PER + i) * 1024 + lane * 16) = w;
        }
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

// Eight outputs from column c on, in one row after another: bias holds the columns' biases,
// and a row's part of the residual is asked for before the row's turn.  A PLAIN epilogue
// only rounds and stores.
template <int F, bool PLAIN>
struct Eight {
    float bias[8];
    s16x8 res;
    __device__ __forceinline__ void init(const ProductArgs& p, int c) {
        if (PLAIN) return;
#pragma unroll
        for (int q = 0; q < 8; ++q) bias[q] = 0.f;
        if (!p.bias || c >= p.cols) return;
        const s16x8 v = row8(p.bias + c, p.cols - c);
#pragma unroll
        for (int q = 0; q < 8; ++q) bias[q] = to_f32<F>((uint16_t)v[q]);
    }
    __device__ __forceinline__ void ask(const ProductArgs& p, int r, int c) {
        if (!PLAIN && p.res && r < p.rows && c < p.cols) res = row8(p.res + (int64_t)r * p.ldr + c, p.cols - c);
    }
    __device__ __forceinline__ void finish(const ProductArgs& p, int r, int c, float (&z)[8], s16x8 rest) const {
        if (r >= p.rows || c >= p.cols) return;
        s16x8 v, k;
        if (!PLAIN) {
#pragma unroll
            for (int q = 0; q < 8; ++q) z[q] += bias[q];
            if (p.z)
#pragma unroll
                for (int q = 0; q < 8; ++q) k[q] = (short)keep_z<F>(z[q]);
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
            if (p.res)
#pragma unroll
                for (int q = 0; q < 8; ++q) z[q] += to_f32<F>((uint16_t)rest[q]);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = (short)to_16<F>(z[q]);
        uint16_t* out = p.out + (int64_t)r * p.ldo + c;
        uint16_t* keep = p.z + (int64_t)r * p.cols + c;
        if (c + 8 <= p.cols) {
            reinterpret_cast<S16x8*>(out)->v = v;
            if (!PLAIN && p.z) reinterpret_cast<S16x8*>(keep)->v = k;
            return;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            if (c + q >= p.cols) break;
            out[q] = (uint16_t)v[q];
            if (!PLAIN && p.z) keep[q] = (uint16_t)k[q];
        }
    }
};

// A wave's 16 x 64 block of sums as the MFMA leaves it (row lane & 15, four columns per
// tile of 16) goes through LDS, so that lanes take eight columns of a row: whole 128-byte
// lines to and from memory.  Its 16-byte places are permuted by the row.
constexpr int EPI_BYTES = 16 * 64 * 4;
// Orders the wave's LDS accesses before and after it: what its lanes wrote is what its lanes
// read next.  No instruction; LDS serves a wave's accesses in the order in which they are issued.
__device__ __forceinline__ void epi_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ void epi_put(char* lds, int lane, int j, f32x4 v) {
    const int r = lane & 15;
    *reinterpret_cast<f32x4*>(lds + r * 256 + (((j * 4 + (lane >> 4)) ^ r) * 16)) = v;
}
__device__ __forceinline__ f32x4 epi_get(const char* lds, int lane, int j) {
    const int r = lane & 15;
    return *reinterpret_cast<const f32x4*>(lds + r * 256 + (((j * 4 + (lane >> 4)) ^ r) * 16));
}
// Finishes two such blocks.
template <int F, bool PLAIN>
__device__ __forceinline__ void epi_rows(const ProductArgs& p, const char* lds, int lane, int r0, int c0, Eight<F, PLAIN>& e) {
    // a forward that has nothing to add: 65.7 us for 2048 x 4096 x 4096, 67.3 through the other
    if (!PLAIN && !p.bias && !p.res && !p.z && p.act == ACT_NONE) {
        Eight<F, true> plain;
        return epi_rows(p, lds, lane, r0, c0, plain);
    }
    const int c = c0 + (lane & 7) * 8;
    e.ask(p, r0 + (lane >> 3), c);
#pragma unroll 4
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (lane >> 3), q = (lane & 7) * 2, m = r & 15;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(lds + r * 256 + ((q ^ m) * 16));
        const f32x4 hi = *reinterpret_cast<const f32x4*>(lds + r * 256 + (((q + 1) ^ m) * 16));
        float z[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        const s16x8 res = e.res;
        if (i < 3) e.ask(p, r0 + r + 8, c);
        e.finish(p, r0 + r, c, z, res);
    }
}

// BM x BN outputs per workgroup, 64 depths a step in two LDS buffers; WM x WN waves.
// The sixteen-wide MFMA takes b's tile as its rows, so a lane ends with four consecutive
// columns of one output row.
//
// Bound by the CU's path from the L2 into LDS: without the operands' loads 4096^3 runs at
// 1940 TFLOP/s, and the loads alone take 60 to 75% of the whole, the same where all tiles read
// the same addresses.  Hence the largest square tile that LDS holds twice (2 x 64 KiB), loads
// that write LDS themselves, the next step's asked for before this one's products, and no
// conflicts in LDS, which is busy 22 to 26% of the time.  bf16, forward, dx, dw, after some
// milliseconds of the same (the clocks settle): 8192^3 1340, 1330 and 1355 TFLOP/s, 4096^3 1305,
// 1308 and 1358, 8192 x 11008 x 4096 600, 552 and 580 us, 2048 x 4096 x 4096 63, 62 and 56 us.
// On a slower card, where 8192^3 ran at 1227, 1285 and 1305, four stages of 32 depths gave 1178
// to 1285, loads through registers 1060 to 1123.
// BITS: b is a palette's.
// E: what becomes of the sums where that is not the epilogue above: E::Args, a ProductArgs, are
// the kernel's; E::begin sets what only the device knows, and says whether there is anything to
// do; an E is made for a wave's rows before the sums are, so that what it reads is there by
// then, and its block takes 16 x 64 sums as the MFMA leaves them.
template <class E, int TR>
struct EndOf {
    typedef typename E::template End<TR> type;
};
template <int TR>
struct EndOf<void, TR> {
    typedef void type;
};
struct NoEnd {
    __device__ __forceinline__ void init(const ProductArgs&, int, int) {}
};
template <int F, int OPA, int OPB, int BM, int BN, int WM, int WN, bool DIRECT, int BITS = 0, class E = void>
__global__ void __launch_bounds__(WM * WN * 64, 2) k_tiled(typename ArgsOf<E>::type p) {
    if constexpr (!std::is_void_v<E>)
        if (!E::begin(p)) return;
    constexpr int NW = WM * WN, TR = BM / WM / 16, TC = BN / WN / 16;
    static_assert(TC == 4 && TR % 4 == 0, "a wave's columns are those of the epilogue");
    typedef Feed<OPA, BM, NW, DIRECT> FA;
    typedef std::conditional_t<BITS == 0, Feed<OPB, BN, NW, DIRECT>, PaletteFeed<F, BITS ? BITS : 1, BN, NW>> FB;
    // four arrays, so that the compiler knows the loads of one buffer apart from the reads of the other
    __shared__ __attribute__((aligned(1024))) char a0[FA::T::BYTES], a1[FA::T::BYTES], b0[FB::T::BYTES], b1[FB::T::BYTES];
    static_assert(NW * 2 * EPI_BYTES <= FA::T::BYTES + FB::T::BYTES, "the epilogue's blocks fit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tx, ty;
    const uint32_t nx = (p.cols + BN - 1) / BN, ny = (p.rows + BM - 1) / BM;
    const uint32_t group = p.first + blockIdx.x, split = group / (nx * ny);
    if constexpr (!std::is_void_v<E>)
        if (split >= (uint32_t)p.splits) return;     // a grid for more rows than there are
    tile_of(group % (nx * ny), nx, ny, tx, ty);
    const int r0 = ty * BM, c0 = tx * BN;
    const int wr = (wave / WN) * (BM / WM), wc = (wave % WN) * (BN / WN);
    FA fa;
    FB fb;
    fa.init(p.a, p.lda, r0, p.rows, p.depth, wave, lane);
    if constexpr (BITS != 0) {
        __shared__ __attribute__((aligned(128))) uint32_t table[FB::TABLE];
        FB::fill(table, p.lut);
        fb.init(p, table, c0, wave, lane);
        fb.load(split * p.split_steps * 64);
        __syncthreads();
    } else {
        fb.init(p.b, p.ldb, c0, p.cols, p.depth, wave, lane);
    }
    std::conditional_t<std::is_void_v<E>, NoEnd, typename EndOf<E, TR>::type> end;
    end.init(p, lane, r0 + wr);
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
            // the SIMD's wave that multiplies before the one that reads (8192 x 32000 x 4096: 1672 -> 1635 us)
            if (!std::is_void_v<E>) __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < TR; ++i)
#pragma unroll
                for (int j = 0; j < TC; ++j) acc[i][j] = mfma16<F>(vb[j], va[i], acc[i][j]);
            if (!std::is_void_v<E>) __builtin_amdgcn_s_setprio(0);
            if (BITS && ks == 0 && s + 1 < steps) fb.finish(bn, (s + 1) * 64);
        }
        if (s + 1 < steps) {
            fa.finish(an, (s + 1) * 64);
            if (!BITS) fb.finish(bn, (s + 1) * 64);
        }
        __syncthreads();
    };
    if (first < steps) {
        fa.start(a0, first * 64);
        fb.start(b0, first * 64);
        fa.finish(a0, first * 64);
        fb.finish(b0, first * 64);
    }
    __syncthreads();
    for (int s = first; s < steps; s += 2) {
        step(a0, b0, a1, b1, s);
        if (s + 1 < steps) step(a1, b1, a0, b0, s + 1);
    }
    if ((BM == SPLIT_TILE || !std::is_void_v<E>) && p.part) {
        float* at = p.part + ((int64_t)group * NW + wave) * (TR * 1024) + lane * 4;
#pragma unroll
        for (int i = 0; i < TR; ++i)
#pragma unroll
            for (int j = 0; j < TC; ++j) *reinterpret_cast<f32x4*>(at + (i * TC + j) * 256) = acc[i][j];
        return;
    }
    // each wave has two blocks of LDS: in a0/a1 the first half of the waves, in b0/b1 the others
    char* mine = (wave < NW / 2 ? a0 : b0) + (wave % (NW / 2)) * 2 * EPI_BYTES;
    if constexpr (!std::is_void_v<E>) {
#pragma unroll
        for (int i = 0; i < TR; ++i) end.block(p, i, mine, lane, r0 + wr + i * 16, c0 + wc, acc[i], ((int64_t)group * NW + wave) * TR + i);
        return;
    }
    Eight<F, OPB == OP_DEPTH> eight;
    eight.init(p, c0 + wc + (lane & 7) * 8);
    static_assert(NW / 2 * 2 * EPI_BYTES <= (FA::T::BYTES < FB::T::BYTES ? FA::T::BYTES : FB::T::BYTES), "");
#pragma unroll
    for (int i = 0; i < TR; i += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < TC; ++j) epi_put(mine + h * EPI_BYTES, lane, j, acc[i + h][j]);
        epi_order();
        epi_rows(p, mine, lane, r0 + wr + i * 16, c0 + wc, eight);
        epi_order();
    }
}

// Adds the partial sums of a split product and finishes them: 16 x 64 outputs per workgroup,
// each of its W waves a part of the splits, one after the other.  Bound by the partial sums'
// bytes for few splits, where one wave is best (512 x 4096 x 4096 in four parts: 29.8 us with
// the product, 30.3 by four waves), and by the chain of loads for many (128 x 128 x 32768 in
// 64: 20.0 us, 14.3 by four).
template <int F, int BM, int BN, int WM, int WN, bool PLAIN, int W, class E = void>
__global__ void __launch_bounds__(W * 64) k_join(typename ArgsOf<E>::type p, int splits) {
    if constexpr (!std::is_void_v<E>) {
        if (!E::begin(p) || p.splits == 1) return;
        splits = p.splits;
    }
    constexpr int NW = WM * WN, TR = BM / WM / 16;
    __shared__ __attribute__((aligned(16))) char lds[W][EPI_BYTES];
    const uint32_t nx = (p.cols + BN - 1) / BN, ny = (p.rows + BM - 1) / BM;
    const uint32_t w = blockIdx.x / (NW * TR);
    const int wave = blockIdx.x / TR % NW, i = blockIdx.x % TR, lane = threadIdx.x & 63, share = threadIdx.x >> 6;
    uint32_t tx, ty;
    if constexpr (!std::is_void_v<E>)
        if (w >= nx * ny) return;
    tile_of(w, nx, ny, tx, ty);
    const int r0 = ty * BM + wave / WN * (BM / WM) + i * 16, c0 = tx * BN + wave % WN * 64;
    if (r0 >= p.rows || c0 >= p.cols) return;
    const int c = (threadIdx.x & 7) * 2;
    Eight<F, PLAIN> eight;
    eight.init(p, c0 + c * 4);
    f32x4 acc[4] = {};
    const float* at = p.part + ((int64_t)w * NW + wave) * (TR * 1024) + i * 1024 + lane * 4;
    const int64_t stride = (int64_t)nx * ny * NW * (TR * 1024);
    const int per = (splits + W - 1) / W, end = min(splits, (share + 1) * per);
#pragma unroll 4
    for (int s = share * per; s < end; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += *reinterpret_cast<const f32x4*>(at + s * stride + j * 256);
    if constexpr (!std::is_void_v<E>) {
        typename EndOf<E, 1>::type end;
        end.init(p, lane, r0);
        if (W > 1) {
            // the waves' shares, by the first wave
#pragma unroll
            for (int j = 0; j < 4; ++j) epi_put(lds[share], lane, j, acc[j]);
            __syncthreads();
            if (share) return;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[j] = f32x4{};
#pragma unroll
                for (int q = 0; q < W; ++q) acc[j] += epi_get(lds[q], lane, j);
            }
            epi_order();
        }
        end.block(p, 0, lds[0], lane, r0, c0, acc, ((int64_t)w * NW + wave) * TR + i);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) epi_put(lds[share], lane, j, acc[j]);
    __syncthreads();
    for (int r = threadIdx.x >> 3; r < 16; r += W * 8) {
        eight.ask(p, r0 + r, c0 + c * 4);
        f32x4 lo = {}, hi = {};
#pragma unroll
        for (int q = 0; q < W; ++q) {
            lo += *reinterpret_cast<const f32x4*>(lds[q] + r * 256 + ((c ^ r) * 16));
            hi += *reinterpret_cast<const f32x4*>(lds[q] + r * 256 + (((c + 1) ^ r) * 16));
        }
        float z[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        eight.finish(p, r0 + r, c0 + c * 4, z, eight.res);
    }
}

template <int F, int OPA, int OPB, int B, int WM, int WN, bool DIRECT, int BITS = 0>
static hipError_t tiled(ProductArgs p, const ProductPlan& q, hipStream_t s) {
    const int64_t tiles = ((int64_t)p.cols + B - 1) / B * (((int64_t)p.rows + B - 1) / B);
    EDKM_GO_PARTS((k_tiled<F, OPA, OPB, B, B, WM, WN, DIRECT, BITS>), (uint64_t)(tiles * q.splits), WM * WN * 64, p);
    if constexpr (B == SPLIT_TILE) {
        const dim3 blocks((uint32_t)(tiles * WM * WN * (B / WM / 16)));
        if (q.splits > 8) EDKM_GO((k_join<F, B, B, WM, WN, OPB == OP_DEPTH, 4>), blocks, dim3(256), p, q.splits);
        else if (q.splits > 1) EDKM_GO((k_join<F, B, B, WM, WN, OPB == OP_DEPTH, 1>), blocks, dim3(64), p, q.splits);
    }
    return hipSuccess;
}

}  // namespace edkm
