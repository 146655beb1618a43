// Products of few tokens with 16-bit or palettized weights, and the 16-bit weights of a
// palette, for gfx950 (MI355X).

#include "edkm_loss.h"

#include <algorithm>
#include <type_traits>

namespace edkm {

// Thirty-two weights per thread, eight at a time, each wave writing whole lines: bound by the
// bytes written.  PAST: by stores past the caches, for weights that nothing reads at once:
// 11008 x 4096 at 3 bits, 107 MB, takes 17.2 us so (6.2 TB/s), 27.2 through them; but the
// product of 512 tokens with the decoded weights then 95 us instead of 82, since it
// finds them there.  Unaligned indices and ragged ends take any alignment.
template <int F, int BITS, bool PAST>
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
            if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<s16x8*>(out + i));
            else *reinterpret_cast<s16x8*>(out + i) = v;
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (i + q < n) out[i + q] = (uint16_t)v[q];
        }
    }
}

// The rows of a matrix (16-bit values, or with BITS a palette's) from rows of any length
// and alignment to rows of whole 16-byte pieces, zeros behind their ends: what the tiled
// products' loads want, for one pass over the operand.  A product of 4097 x 4095 x 4097 takes
// 229, 193 and 201 us (forward, dx, dw) with the copies and 311, 319 and 585 without, and even
// 1001 x 1333 x 777 gains (21.2, 22.6 and 24.6 against 24.1, 28.3 and 61.6).  Up to three matrices
// a launch, one of them per blockIdx.y.
template <int F, int BITS>
__global__ void __launch_bounds__(256) k_align_rows(AlignArgs a, const uint8_t* idx, uint64_t nbytes, const float* lut) {
    Decoder<F> dec;
    if constexpr (BITS != 0) dec.init(lut, BITS);
    const AlignJob& job = a.job[BITS ? 0 : blockIdx.y];
    const uint16_t* m = job.m;
    uint16_t* out = job.out;
    const int64_t ld = job.ld;
    const int cols = job.cols;
    const uint32_t pieces = ((uint32_t)cols + 7) / 8;
    const uint64_t total = (uint64_t)job.rows * pieces;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256) {
        const uint32_t r = (uint32_t)(i / pieces), c = (uint32_t)(i % pieces) * 8;
        const int left = cols - (int)c;
        s16x8 v;
        if constexpr (BITS != 0)
            v = keep_first(dec.eight(load_idx8(idx, nbytes, (uint64_t)r * (uint32_t)cols + c, BITS), BITS), left);
        else
            v = row8(m + (int64_t)r * ld + c, left);
        *reinterpret_cast<s16x8*>(out + i * 8) = v;
    }
}

// ----------------------------------------------------------------------------
// products of few tokens

// A lane's weights of a run: 32 depths of one row, as 16-bit values (BITS 0) or as packed
// indices.  WHOLE: 32 depths are 4 BITS bytes on a 4-byte boundary (16-bit values: 64 bytes
// on a 16-byte one), and offsets from the workgroup's first row fit 32 bits; else any
// alignment and end.
template <int F, int BITS, bool WHOLE>
struct FewWeights {
    uint32_t raw[BITS ? 4 : 1];
    s16x8 w[BITS ? 1 : 4];

    // `at`: the run's bytes of the first row (the same for all lanes), `off`: the lane's from there
    __device__ __forceinline__ void load_whole(const char* at, uint32_t off) {
        if constexpr (BITS == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const s16x8*>(at + off + j * 16);
        } else {
#pragma unroll
            for (int j = 0; j < BITS; ++j) raw[j] = *reinterpret_cast<const uint32_t*>(at + off + j * 4);
        }
    }
    __device__ __forceinline__ void load_any(const ProductArgs& p, int row, int d) {
        const int left = p.depth - d;
        if constexpr (BITS == 0) {
            const uint16_t* at = p.b + (int64_t)row * p.ldb + d;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = row8(at + j * 8, left - j * 8);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                raw[j] = left > j * 8 ? load_idx8(p.idx, p.idx_bytes, (uint64_t)row * (uint32_t)p.depth + d + j * 8, BITS) : 0;
        }
    }
    // the values of depths 8 j .. 8 j + 7
    __device__ __forceinline__ s16x8 eight(const char* mine, int j) const {
        if constexpr (BITS == 0) {
            return w[j];
        } else {
            typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
            uint32_t v;
            if (WHOLE) {
                constexpr int BPJ = 8 * BITS;                 // bits of eight indices
                const int at = j * BPJ, q = at / 32, sh = at % 32;
                v = sh + BPJ > 32 ? __builtin_amdgcn_alignbit(raw[q + 1 < 4 ? q + 1 : 3], raw[q], sh) : sh ? raw[q] >> sh : raw[q];
            } else {
                v = raw[j];
            }
            u32x4 r;
            constexpr uint32_t MASK = ((1u << (2 * BITS)) - 1) * (PAIR_BANKS * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int sh = 2 * BITS * i - 7;              // the pair times 128 bytes
                const uint32_t e = (sh < 0 ? v << (sh < 0 ? -sh : 0) : v >> (sh < 0 ? 0 : sh)) & MASK;
                r[i] = *reinterpret_cast<const uint32_t*>(mine + e);
            }
            return __builtin_bit_cast(s16x8, r);
        }
    }
};

// Up to 16 MT tokens against 16 NT weight rows per workgroup.  The waves share the depths by
// runs of 128 and add their sums through LDS.  The MFMA takes the weights as its rows: lane
// l holds row l mod 16, depths 32 (l / 16) + 8 j + 0 .. 7 of a run at its j-th step, so its
// share of a palette's run is 4 b consecutive bytes.  A wave asks for its weights of U runs,
// and for U more ahead, before it waits for anything, the table included.  One
// token's 16-bit weights are bound by their bytes.  With a palette it is the chain of a
// workgroup's steps: with 11008 depths at 4 bits the vector units are busy for 29% of the time,
// LDS for 19%, and the waves wait for loads and barriers for 59% of theirs, with one workgroup
// of sixteen waves on a CU and five or six runs a wave.  Addresses are one 32-bit offset per row
// from a pointer that all lanes share.  More tokens are bound by their way into the CUs, since
// every workgroup reads all of them: 64 x 4096 are 512 KiB each, 12 bytes a clock.  A call among
// others takes, with 3 bits and 4096 depths, for 4096 outputs 5.1 us (1 token), 7.4 (16), 18.1
// (64); for 11008 outputs 8.1 (2.1 TB/s of indices), 10.3 and 22.9; 16-bit weights of 11008
// outputs 18.6 us (4.8 TB/s).
// E: what becomes of the sums where that is not the epilogue; its row16 takes sixteen of a row.
template <int F, int BITS, bool WHOLE, int MT, int NT, int U, int NW, class E = void>
__global__ void __launch_bounds__(NW * 64) k_few(typename ArgsOf<E>::type p) {
    constexpr int ENTRIES = 1 << (2 * BITS);
    constexpr int TABLE = BITS ? ENTRIES * PAIR_BANKS : 0, SUMS = NW * MT * NT * 256;
    // the table, and after the last lookup the waves' sums
    __shared__ __attribute__((aligned(128))) uint32_t lds[TABLE > SUMS ? TABLE : SUMS];
    __shared__ uint16_t tab[KMAX];
    uint32_t* pairs = lds;
    float* red = reinterpret_cast<float*>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int l = lane & 15, g = lane >> 4;
    const int c0 = (p.first + blockIdx.x) * 16 * NT;
    const int runs = (p.depth + 127) / 128;
    constexpr int RUN_BYTES = BITS ? 16 * BITS : 256;        // of one row
    const uint32_t row_bytes = BITS ? (uint32_t)((uint64_t)p.depth * BITS / 8) : (uint32_t)(p.ldb * 2);
    const char* wat = BITS ? reinterpret_cast<const char*>(p.idx) + (uint64_t)c0 * row_bytes
                           : reinterpret_cast<const char*>(p.b) + (int64_t)c0 * p.ldb * 2;
    FewWeights<F, BITS, WHOLE> now[U][NT], next[BITS ? U : 1][BITS ? NT : 1];
    s16x8 x[U][MT][4];
    uint32_t woff[NT], xoff[MT];
    int row[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        row[n] = min(c0 + n * 16 + l, p.cols - 1);
        woff[n] = (uint32_t)(row[n] - c0) * row_bytes + g * (RUN_BYTES / 4);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) xoff[i] = (uint32_t)(min(i * 16 + l, p.rows - 1) * (int)p.lda + g * 32) * 2;
    // Depths past the end (WHOLE: all 32 of a lane, in the last run): the lane reads the
    // run's first ones instead, and its values are cleared before the product.
    auto back = [&](int t) { return t * 128 + 128 > p.depth && t * 128 + g * 32 >= p.depth; };
    auto load_x = [&](int t0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = min(t0 + u * nw, runs - 1);
            const bool b = back(t);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                // lanes without a token load nothing (their columns are not used): what a load costs is its lanes
                if (i * 16 + l >= p.rows) continue;
                if constexpr (WHOLE) {
                    const char* at = reinterpret_cast<const char*>(p.a) + (int64_t)t * 256;
                    const uint32_t off = xoff[i] - (b ? g * 64 : 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[u][i][j] = *reinterpret_cast<const s16x8*>(at + off + j * 16);
                } else {
                    const int d = t * 128 + g * 32;
                    const uint16_t* at = p.a + (int64_t)(i * 16 + l) * p.lda + d;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[u][i][j] = row8(at + j * 8, p.depth - d - j * 8);
                }
            }
        }
    };
    auto load_w = [&](auto& to, int t0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = min(t0 + u * nw, runs - 1);
            const bool b = back(t);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (WHOLE) to[u][n].load_whole(wat + (int64_t)t * RUN_BYTES, woff[n] - (b ? g * (RUN_BYTES / 4) : 0));
                else to[u][n].load_any(p, row[n], t * 128 + g * 32);
            }
        }
    };
    load_w(now, wave);
    load_x(wave);
    if constexpr (BITS != 0) {
        if (threadIdx.x < (1 << BITS)) tab[threadIdx.x] = to_16<F>(p.lut[threadIdx.x]);
        __syncthreads();
        for (int i = threadIdx.x; i < ENTRIES * PAIR_BANKS; i += blockDim.x) {
            const int e = i / PAIR_BANKS;
            pairs[i] = (uint32_t)tab[e & ((1 << BITS) - 1)] | ((uint32_t)tab[e >> BITS] << 16);
        }
        __syncthreads();
    }
    const char* mine = reinterpret_cast<const char*>(pairs + (lane & (PAIR_BANKS - 1)));
    f32x4 acc[MT][NT] = {};
    // one run; TAIL: only the lane's first `left` depths count (WHOLE: all or none)
    auto run = [&](int u, int left, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s16x8 xj[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                xj[i] = x[u][i][j];
                if (TAIL) xj[i] = WHOLE ? (left > 0 ? xj[i] : s16x8{}) : keep_first(xj[i], left - j * 8);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s16x8 w = now[u][n].eight(mine, j);
                if (TAIL) w = WHOLE ? (left > 0 ? w : s16x8{}) : keep_first(w, left - j * 8);
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i][n] = mfma16<F>(w, xj[i], acc[i][n]);
            }
        }
    };
    for (int t = wave; t < runs; t += nw * U) {
        const bool more = t + nw * U < runs;
        if constexpr (BITS != 0)
            if (more) load_w(next, t + nw * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int tu = t + u * nw;
            if (tu * 128 + 128 <= p.depth) run(u, 0, std::false_type{});
            else if (tu < runs) run(u, p.depth - (tu * 128 + g * 32), std::true_type{});
        }
        if (more) {
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
    if (BITS) __syncthreads();
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
        if constexpr (!std::is_void_v<E>) {
            E::row16(p, r, col, z);
            continue;
        }
        if (col >= p.cols) continue;
        if (p.bias) z += to_f32<F>(p.bias[col]);
        if (p.z) p.z[(int64_t)r * p.cols + col] = keep_z<F>(z);
        float y = act_value(z, p.act);
        if (p.res) y += to_f32<F>(p.res[(int64_t)r * p.ldr + col]);
        p.out[(int64_t)r * p.ldo + col] = to_16<F>(y);
    }
}

template <int F, int BITS, bool WHOLE, int MT, int NT, class E = void>
static hipError_t few_go(typename ArgsOf<E>::type p, hipStream_t s) {
    constexpr int U = WHOLE && BITS && MT == 1 && NT < 3 ? 2 : 1, NW = MT == 1 ? 16 : 8;
    const int runs = (p.depth + 127) / 128;
    int nw = 1;
    while (nw < runs && nw < NW) nw *= 2;
    EDKM_GO_PARTS((k_few<F, BITS, WHOLE, MT, NT, U, NW, E>), ((uint64_t)p.cols + 16 * NT - 1) / (16 * NT), nw * 64, p);
    return hipSuccess;
}

// Weight rows of a workgroup, in sixteens.  More of them share the reading of the tokens and
// the making of the table, and cost a workgroup time: 1.5 and 2 times one's for up to 16
// tokens, 1.13 and 1.25 times for more.  So the number whose rounds over the CUs take least
// (3 bits, 4096 depths, us with 16, 32 and 48 rows: one token and 8192 outputs 8.2, 6.7, -,
// 11008 11.0, 11.4, 8.1, 16384 14.3, 11.8, 14.1; 32 tokens and 11008 26.6, 21.7, 14.2, 16384
// 34.7, 21.9, 26.1).  A few tokens' 16-bit weights, bound by their bytes, want many small
// workgroups (one token and 11008 outputs 18.6, 26.5).
template <int F, int BITS, bool WHOLE, int MT>
static hipError_t few_rows(const ProductArgs& p, hipStream_t s) {
    if constexpr (!WHOLE || (MT == 1 && BITS == 0)) {
        return few_go<F, BITS, WHOLE, MT, 1>(p, s);
    } else {
        const int64_t tiles = ((int64_t)p.cols + 15) / 16;
        auto time = [&](int64_t n) { return ((tiles + n - 1) / n + 255) / 256 * ((MT == 1 ? 1 : 7) + n); };
        if (time(1) <= time(2) && time(1) <= time(3)) return few_go<F, BITS, WHOLE, MT, 1>(p, s);
        return time(2) <= time(3) ? few_go<F, BITS, WHOLE, MT, 2>(p, s) : few_go<F, BITS, WHOLE, MT, 3>(p, s);
    }
}

template <int F, int BITS, bool WHOLE>
static hipError_t few_bits(const ProductArgs& p, hipStream_t s) {
    if (p.rows <= 16) return few_rows<F, BITS, WHOLE, 1>(p, s);
    return p.rows <= 32 ? few_rows<F, BITS, WHOLE, 2>(p, s) : few_rows<F, BITS, WHOLE, 4>(p, s);
}

static bool few_whole(const ProductArgs& p, int bits) {
    // 32-bit offsets: 64 rows of at most 2^25 bytes
    const bool x16 = ((uintptr_t)p.a & 15) == 0 && p.lda % 8 == 0 && p.depth % 32 == 0 && p.lda < (1 << 24) && p.ldb < (1 << 24);
    return x16 && (bits ? ((uintptr_t)p.idx & 3) == 0 : ((uintptr_t)p.b & 15) == 0 && p.ldb % 8 == 0);
}

template <int F>
static hipError_t few(const ProductArgs& p, int bits, hipStream_t s) {
    const bool whole = few_whole(p, bits);
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

hipError_t launch_few_loss(const LossArgs& p, int fmt, hipStream_t s) {
    const bool whole = few_whole(p, 0);
    if (fmt == FMT_BF16) return whole ? few_go<FMT_BF16, 0, true, 1, 1, LossStats>(p, s) : few_go<FMT_BF16, 0, false, 1, 1, LossStats>(p, s);
    return whole ? few_go<FMT_FP16, 0, true, 1, 1, LossStats>(p, s) : few_go<FMT_FP16, 0, false, 1, 1, LossStats>(p, s);
}

template <int F, bool PAST>
static hipError_t unpalettize_f(const uint8_t* idx, uint64_t nb, uint64_t n, int bits, const float* lut, uint16_t* out,
                                hipStream_t s) {
    const dim3 grid((uint32_t)((n + 8191) / 8192));
    const int al = ((uintptr_t)out & 15) == 0;
    if (bits == 1) EDKM_GO((k_unpalettize<F, 1, PAST>), grid, dim3(256), idx, nb, n, lut, out, al);
    else if (bits == 2) EDKM_GO((k_unpalettize<F, 2, PAST>), grid, dim3(256), idx, nb, n, lut, out, al);
    else if (bits == 3) EDKM_GO((k_unpalettize<F, 3, PAST>), grid, dim3(256), idx, nb, n, lut, out, al);
    else EDKM_GO((k_unpalettize<F, 4, PAST>), grid, dim3(256), idx, nb, n, lut, out, al);
    return hipSuccess;
}

hipError_t launch_unpalettize(const uint8_t* idx, uint64_t idx_bytes, uint64_t n, int bits, int fmt, const float* lut,
                              uint16_t* out, bool past, hipStream_t s) {
    if (past)
        return fmt == FMT_BF16 ? unpalettize_f<FMT_BF16, true>(idx, idx_bytes, n, bits, lut, out, s)
                               : unpalettize_f<FMT_FP16, true>(idx, idx_bytes, n, bits, lut, out, s);
    return fmt == FMT_BF16 ? unpalettize_f<FMT_BF16, false>(idx, idx_bytes, n, bits, lut, out, s)
                           : unpalettize_f<FMT_FP16, false>(idx, idx_bytes, n, bits, lut, out, s);
}

static uint32_t align_grid(int64_t rows, int64_t cols) {
    return (uint32_t)std::min<int64_t>((rows * ((cols + 7) / 8) + 255) / 256, 8192);
}

hipError_t launch_align_rows(const AlignArgs& a, hipStream_t s) {
    if (a.count == 0) return hipSuccess;
    uint32_t grid = 1;
    for (int i = 0; i < a.count; ++i) grid = std::max(grid, align_grid(a.job[i].rows, a.job[i].cols));
    EDKM_GO((k_align_rows<FMT_BF16, 0>), dim3(grid, a.count), dim3(256), a, (const uint8_t*)nullptr, (uint64_t)0, (const float*)nullptr);
    return hipSuccess;
}

template <int F>
static hipError_t unpalettize_rows_f(const uint8_t* idx, uint64_t nb, int rows, int cols, int bits, const float* lut, uint16_t* out,
                                     hipStream_t s) {
    const dim3 grid(align_grid(rows, cols));
    AlignArgs a{};
    a.job[0] = {nullptr, 0, rows, cols, out};
    if (bits == 1) EDKM_GO((k_align_rows<F, 1>), grid, dim3(256), a, idx, nb, lut);
    else if (bits == 2) EDKM_GO((k_align_rows<F, 2>), grid, dim3(256), a, idx, nb, lut);
    else if (bits == 3) EDKM_GO((k_align_rows<F, 3>), grid, dim3(256), a, idx, nb, lut);
    else EDKM_GO((k_align_rows<F, 4>), grid, dim3(256), a, idx, nb, lut);
    return hipSuccess;
}

hipError_t launch_unpalettize_rows(const uint8_t* idx, uint64_t nb, int64_t rows, int64_t cols, int bits, int fmt, const float* lut,
                                   uint16_t* out, hipStream_t s) {
    return fmt == FMT_BF16 ? unpalettize_rows_f<FMT_BF16>(idx, nb, (int)rows, (int)cols, bits, lut, out, s)
                           : unpalettize_rows_f<FMT_FP16>(idx, nb, (int)rows, (int)cols, bits, lut, out, s);
}

}  // namespace edkm
