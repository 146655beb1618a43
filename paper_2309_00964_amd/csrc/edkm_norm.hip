// The step from one block to the next, for gfx950 (MI355X): the norm of a block's output,
// its gate and scale, the residual addition and the next block's norm in one pass, and the
// gradients of all of them in another.

#include "edkm_model.h"
#include "edkm_product.h"

#include <algorithm>

namespace edkm {

// The sum of a wave's values, by moves between lanes of a row of sixteen and from row to row.
template <int MOVE, int ROWS>
__device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), MOVE, ROWS, 0xF, false));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0x111, 0xF>(v);      // row_shr:1, 2, 4, 8: the last lane of a row has its sum
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);      // row_bcast:15 and 31: the last lane has all rows'
    v += moved<0x143, 0xC>(v);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// The same of sixteen lanes, in all of them, and of a row of lanes and the next one's.
__device__ __forceinline__ float row_sum(float v) {
    v += moved<0xB1, 0xF>(v);       // lanes in pairs, pairs in fours, fours and eights mirrored
    v += moved<0x4E, 0xF>(v);
    v += moved<0x141, 0xF>(v);
    return v + moved<0x140, 0xF>(v);
}
__device__ __forceinline__ float two_rows(float v) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float two_halves(float v) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// L threads share a row, each with I pieces of eight columns.
template <int L>
struct Row {
    static constexpr int THREADS = L <= 64 ? 256 : L;
    static constexpr int ROWS = THREADS / L;      // of a workgroup, side by side
    static constexpr int WAVES = L / 64;

    // The thread's row among its workgroup's; where it is the same for a wave its addresses are scalars.
    __device__ __forceinline__ static uint32_t mine() {
        return ROWS == 1 ? 0 : L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : threadIdx.x / L;
    }

    // Sums of a row's K values over its threads.  Sums that follow one another take different
    // places in LDS, so that one barrier each is enough.
    template <int K>
    __device__ __forceinline__ static void sum(float (&v)[K], float (*lds)[16], int place) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = L == 16 ? row_sum(v[k]) : L == 32 ? two_rows(row_sum(v[k])) : wave_sum(v[k]);
        if constexpr (WAVES > 1) {
            static_assert(WAVES <= 16 && K <= 3, "places");
            const int w = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) lds[place * 3 + k][w] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = 0.f;
#pragma unroll
                for (int q = 0; q < WAVES; ++q) v[k] += lds[place * 3 + k][q];
            }
        }
    }
};

template <int F>
__device__ __forceinline__ void floats(s16x8 v, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = to_f32<F>((uint16_t)v[j]);
}
template <int F, bool PAST = false>
__device__ __forceinline__ void put8(uint16_t* q, const float (&f)[8], int left) {
    s16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (short)to_16<F>(f[j]);
    if (left >= 8) {
        typedef short any8 __attribute__((ext_vector_type(8), aligned(2)));
        if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<any8*>(q));
        else reinterpret_cast<S16x8*>(q)->v = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) q[j] = (uint16_t)v[j];
}

// Keeps a vector's values as they are: without it the compiler converts them once before the
// loop over the rows and holds twice the registers (170 against 117 in k_norm_grad).
__device__ __forceinline__ void packed(s16x8& v) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    u32x4 b = __builtin_bit_cast(u32x4, v);
    asm volatile("" : "+v"(b));
    v = __builtin_bit_cast(s16x8, b);
}

template <int F>
__device__ __forceinline__ s16x8 ones() {
    const short o = F == FMT_BF16 ? 0x3F80 : 0x3C00;
    return s16x8{o, o, o, o, o, o, o, o};
}

__device__ __forceinline__ float over_root(float sum, const NormArgs& a) {
    return __builtin_amdgcn_rsqf(fmaf(sum, 1.0f / (float)a.n, a.eps));
}

// A row lies in its threads' registers from its loads to its stores; the vectors stay there
// from row to row.  Bound by its bytes: r, u (and a gate's) read, h and y written, once: 8192 x 4096
// takes 45 us (6.0 TB/s), one row 3.2.
template <int F, int L, int I, bool BLOCK, bool TINY>
__global__ void __launch_bounds__(Row<L>::THREADS) k_norm(NormArgs a) {
    typedef Row<L> R;
    const bool ragged = a.n % 8 != 0;
    __shared__ float lds[6][16];
    const int l = threadIdx.x % L;
    s16x8 w[I], post[I] = {}, gate[I] = {};
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = (i * L + l) * 8;
        w[i] = row8(a.w + c, a.n - c);
        if (BLOCK && a.post) post[i] = row8(a.post + c, a.n - c);
        if (BLOCK && a.gate && !a.gate_rows) gate[i] = row8(a.gate + c, a.n - c);
    }
    for (int64_t r = (int64_t)blockIdx.x * R::ROWS + R::mine(); r < a.m; r += (int64_t)gridDim.x * R::ROWS) {
        float h[I][8];
        s16x8 nr[I], nu[BLOCK ? I : 1], ng[BLOCK ? I : 1];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8;
            nr[i] = ask8<TINY>(a.r + r * a.ldr, c, a.n);
            if constexpr (BLOCK) {
                nu[i] = ask8<TINY>(a.u + r * a.ldu, c, a.n);
                if (a.gate_rows) ng[i] = ask8<TINY>(a.gate + r * a.ldg, c, a.n);
            }
        }
#pragma unroll
        for (int i = 0; i < I; ++i) floats<F>(had8<TINY>(nr[i], a.n - (i * L + l) * 8, ragged), h[i]);
        if constexpr (BLOCK) {
            float b[I][8], ss[1] = {0.f};
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int c = (i * L + l) * 8;
                floats<F>(had8<TINY>(nu[i], a.n - c, ragged), b[i]);
                if (a.gate_rows) gate[i] = had8<TINY>(ng[i], a.n - c, ragged);
            }
            if (a.post) {
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) ss[0] = fmaf(b[i][j], b[i][j], ss[0]);
                R::sum(ss, lds, 0);
                const float su = over_root(ss[0], a);
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) b[i][j] *= su * to_f32<F>((uint16_t)post[i][j]);
            }
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int c = (i * L + l) * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = a.gate ? a.scale * to_f32<F>((uint16_t)gate[i][j]) : a.scale;
                    h[i][j] = fmaf(g, b[i][j], h[i][j]);
                }
                put8<F>(a.h + r * a.ldh + c, h[i], a.n - c);
            }
        }
        float ss[1] = {0.f};
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) ss[0] = fmaf(h[i][j], h[i][j], ss[0]);
        }
        R::sum(ss, lds, 1);
        const float sh = over_root(ss[0], a);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] *= sh * to_f32<F>((uint16_t)w[i][j]);
            put8<F>(a.y + r * a.ldy + c, h[i], a.n - c);
        }
        if (R::WAVES > 1 && (!BLOCK || !a.post)) __syncthreads();    // place 1 is free for the next row
    }
}

// The gradients, a row in registers as above: dh' = dh + s (g - hn mean(g hn)) with g = dy w,
// hn = s h; then the block's share of it through gate and norm.  h is formed again from r and u,
// which costs no more bytes than reading it and keeps it unrounded.  A thread adds up its
// columns' shares of the vectors' gradients in fp32 over its rows, and k_norm_join the threads':
// dy hn for dw, and one sum for both others, since of scale gate dh' un (dpost) and
// scale dh' un post (a vector gate's) all but dh' un is the column's.  Bound by its bytes and by
// the row's three sums, which wait for one another: 8192 x 4096 with all gradients takes 80 us (5.0
// TB/s), 67 without norm and gate of the block; from 4097 columns on a CU has one workgroup (8192 x
// 8192 177 us, 4.5 TB/s).  PAST: rows are read and written past the caches, where they do not fit
// them (8192 x 4096 90 us through them).
template <int F, int L, int I, bool BLOCK, bool TINY, bool PAST>
__global__ void __launch_bounds__(Row<L>::THREADS, 4) k_norm_grad(NormArgs a) {
    typedef Row<L> R;
    const bool ragged = a.n % 8 != 0;
    // registers for the next row's loads beside this one's work, and for h between its sums
    constexpr bool AHEAD = I == 1;
    __shared__ float lds[9][16];
    const int l = threadIdx.x % L;
    const float per = 1.0f / (float)a.n;
    float sw[I][8] = {}, sb[BLOCK ? I : 1][8] = {};
    const uint32_t group = blockIdx.x * R::ROWS + R::mine(), stride = L < 64 ? gridDim.x * R::ROWS : a.groups;
    s16x8 w[I], post[I] = {}, gate[I] = {};
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = (i * L + l) * 8;
        w[i] = row8(a.w + c, a.n - c);
        // a norm or a gate that is not there is one of ones
        if (BLOCK) post[i] = a.post ? row8(a.post + c, a.n - c) : ones<F>();
        if (BLOCK && !a.gate_rows) gate[i] = a.gate ? row8(a.gate + c, a.n - c) : ones<F>();
    }
    s16x8 nr[I], ndy[I], ndh[I], nu[BLOCK ? I : 1];      // the next row
    auto ask = [&](int64_t r) {
        // where a gradient is not given any row is loaded, and taken as zeros
        const uint16_t *pr = a.r + r * a.ldr, *py = a.dy ? a.dy + r * a.lddy : pr, *ph = a.dh ? a.dh + r * a.lddh : pr;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8;
            nr[i] = ask8<TINY, PAST>(pr, c, a.n);
            ndy[i] = ask8<TINY, PAST>(py, c, a.n);
            ndh[i] = ask8<TINY, PAST>(ph, c, a.n);
            if constexpr (BLOCK) nu[i] = ask8<TINY, PAST>(a.u + r * a.ldu, c, a.n);
        }
    };
    // the row's own: values are taken from 16 bits again for each of its three sums, which leaves
    // the registers for the rows to come
    s16x8 x[I], y[I], z[I], u[I];
    auto again = [&] {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            packed(x[i]);
            packed(y[i]);
            packed(z[i]);
            packed(w[i]);
            if (BLOCK) {
                packed(u[i]);
                packed(post[i]);
                packed(gate[i]);
            }
        }
    };
    if (AHEAD && group < a.m) ask(group);
    for (int64_t r = group; r < a.m; r += stride) {
        if (!AHEAD) ask(r);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8, left = a.n - c;
            if constexpr (BLOCK)
                if (a.gate_rows) gate[i] = had8<TINY>(ask8<TINY>(a.gate + r * a.ldg, c, a.n), left, ragged);
            x[i] = had8<TINY>(nr[i], left, ragged);
            y[i] = a.dy ? had8<TINY>(ndy[i], left, ragged) : s16x8{};
            z[i] = a.dh ? had8<TINY>(ndh[i], left, ragged) : s16x8{};
            if constexpr (BLOCK) u[i] = had8<TINY>(nu[i], left, ragged);
        }
        if (AHEAD && r + stride < a.m) ask(r + stride);
        again();
        float su = 1.f;
        if (BLOCK && a.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float uv = to_f32<F>((uint16_t)u[i][j]);
                    s[0] = fmaf(uv, uv, s[0]);
                }
            R::sum(s, lds, 0);
            su = over_root(s[0], a);
            again();
        }
        // h, as the forward had it
        auto formed = [&](int i, int j) {
            const float v = to_f32<F>((uint16_t)x[i][j]);
            if (!BLOCK) return v;
            const float g = a.scale * to_f32<F>((uint16_t)gate[i][j]), p = su * to_f32<F>((uint16_t)post[i][j]);
            return fmaf(g, to_f32<F>((uint16_t)u[i][j]) * p, v);
        };
        float s[2] = {0.f, 0.f}, s2[1] = {0.f}, h[AHEAD ? I : 1][8];
#pragma unroll
        for (int i = 0; i < I; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = formed(i, j);
                if (AHEAD) h[i][j] = v;
                s[0] = fmaf(v, v, s[0]);
                s[1] = fmaf(to_f32<F>((uint16_t)y[i][j]) * to_f32<F>((uint16_t)w[i][j]), v, s[1]);
            }
        }
        R::sum(s, lds, 1);
        again();
        const float sh = over_root(s[0], a), mean = s[1] * sh * per;
        float q[BLOCK ? I : 1][8];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8;
            float d[8], dg[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float hn = (AHEAD ? h[i][j] : formed(i, j)) * sh, dy = to_f32<F>((uint16_t)y[i][j]);
                d[j] = fmaf(sh, fmaf(-hn, mean, dy * to_f32<F>((uint16_t)w[i][j])), to_f32<F>((uint16_t)z[i][j]));
                sw[i][j] = fmaf(dy, hn, sw[i][j]);
                if constexpr (BLOCK) {
                    const float un = to_f32<F>((uint16_t)u[i][j]) * su, p = a.scale * to_f32<F>((uint16_t)post[i][j]);
                    const float g = to_f32<F>((uint16_t)gate[i][j]);
                    dg[j] = d[j] * un;
                    sb[i][j] = fmaf(dg[j], a.gate_rows ? g : 1.f, sb[i][j]);
                    dg[j] *= p;
                    q[i][j] = d[j] * (g * p);
                    s2[0] = fmaf(q[i][j], un, s2[0]);
                }
            }
            if (a.dr) put8<F, PAST>(a.dr + r * a.lddr + c, d, a.n - c);
            if (BLOCK && a.dgate && a.gate_rows) put8<F>(a.dgate + r * a.n + c, dg, a.n - c);
        }
        if (BLOCK && a.post) R::sum(s2, lds, 2);
        else if (R::WAVES > 1) __syncthreads();      // place 1 is free for the next row
        if (BLOCK && a.du) {
            const float mean2 = a.post ? s2[0] * per : 0.f;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int c = (i * L + l) * 8;
                packed(u[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) q[i][j] = su * fmaf(-to_f32<F>((uint16_t)u[i][j]) * su, mean2, q[i][j]);
                put8<F, PAST>(a.du + r * a.lddu + c, q[i], a.n - c);
            }
        }
    }
    // a wave's rows make one part
    uint32_t at = group;
    if (L < 64) {
        at = blockIdx.x * 4 + (threadIdx.x >> 6);
        auto all = [](float v) { return two_halves(L == 16 ? two_rows(v) : v); };
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sw[0][j] = all(sw[0][j]);
            if (BLOCK) sb[0][j] = all(sb[0][j]);
        }
        if ((threadIdx.x & 63) >= L) return;
    }
    if (at >= a.groups) return;
    auto keep = [&](int k, const float (&v)[8], int c) {
        float* q = a.part + ((int64_t)at * 2 + k) * a.n + c;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < a.n) q[j] = v[j];
    };
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = (i * L + l) * 8;
        if (a.dw) keep(0, sw[i], c);
        if constexpr (BLOCK)
            if (a.dpost || (a.dgate && !a.gate_rows)) keep(1, sb[i], c);
    }
}

// 32 columns of one vector per workgroup, their parts shared by 32 threads each
template <int F>
__global__ void __launch_bounds__(1024) k_norm_join(NormArgs a) {
    __shared__ float red[32][33];
    const int k = blockIdx.y;
    uint16_t *gate = a.gate_rows ? nullptr : a.dgate, *post = a.dpost;
    if (k == 0 ? !a.dw : !gate && !post) return;
    const int l = threadIdx.x & 31, q = threadIdx.x >> 5, c = blockIdx.x * 32 + l;
    float sum = 0.f;
    if (c < a.n)
#pragma unroll 4
        for (uint32_t i = q; i < a.groups; i += 32) sum += a.part[((int64_t)i * 2 + k) * a.n + c];
    red[q][l] = sum;
    __syncthreads();
    sum = red[l][q];
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor(sum, o, 32);
    const int mine = blockIdx.x * 32 + q;
    if (l || mine >= a.n) return;
    if (k == 0) {
        a.dw[mine] = to_16<F>(sum);
        return;
    }
    sum *= a.scale;
    const bool any = a.groups > 0;      // a sum of no rows is 0, whatever it would be a multiple of
    if (post) post[mine] = to_16<F>(any && a.gate && !a.gate_rows ? sum * to_f32<F>(a.gate[mine]) : sum);
    if (gate) gate[mine] = to_16<F>(any && a.post ? sum * to_f32<F>(a.post[mine]) : sum);
}

// ----------------------------------------------------------------------------
// launches

// Threads and pieces of a row by its length, forward and backward (whose sums over the rows
// take two registers a column).  Narrow rows, a head's say, lie side by side in a wave: 65536 x 256 with
// a gate for each value takes 27 and 51 us, by a wave to a row 31 and 96.
template <class Go>
static hipError_t by_length_back(int64_t n, Go go) {
    if (n <= 128) return go(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (n <= 256) return go(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    if (n <= 512) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (n <= 1024) return go(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
    if (n <= 2048) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (n <= 4096) return go(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
    if (n <= 8192) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
    return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}
template <class Go>
static hipError_t by_length(int64_t n, Go go) {
    if (n <= 128) return go(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (n <= 256) return go(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    if (n <= 512) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (n <= 1024) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    if (n <= 2048) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (n <= 4096) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    if (n <= 8192) return go(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
    return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}

// Parts of a backward's sums: one for each row that is in work, or for each wave of narrow rows (up
// to 256 values).  That is two workgroups of four waves a CU up to 512 values, and above them as many
// workgroups, one to a row, as hold 1024 threads of a CU: eight, four, two, one.
uint32_t norm_groups(int64_t m, int64_t n) {
    if (n <= 256) {
        const int64_t rows = n <= 128 ? Row<16>::ROWS : Row<32>::ROWS;
        return (uint32_t)std::min<int64_t>((m + rows - 1) / rows, 512) * 4;
    }
    return (uint32_t)std::min<int64_t>(m, n <= 1024 ? 2048 : n <= 2048 ? 1024 : n <= 4096 ? 512 : 256);
}

template <int F>
static hipError_t norm_f(const NormArgs& a, hipStream_t s) {
    return by_length(a.n, [&](auto L, auto I) -> hipError_t {
        constexpr int l = decltype(L)::value, i = decltype(I)::value;
        const dim3 grid((uint32_t)std::min<int64_t>((a.m + Row<l>::ROWS - 1) / Row<l>::ROWS, 2048)), block(Row<l>::THREADS);
        if (l == 16 && a.n < 8) {
            if (a.u) EDKM_GO((k_norm<F, 16, 1, true, true>), grid, block, a);
            else EDKM_GO((k_norm<F, 16, 1, false, true>), grid, block, a);
        } else if (a.u) {
            EDKM_GO((k_norm<F, l, i, true, false>), grid, block, a);
        } else {
            EDKM_GO((k_norm<F, l, i, false, false>), grid, block, a);
        }
        return hipSuccess;
    });
}

template <int F>
static hipError_t grad_f(const NormArgs& a, hipStream_t s) {
    if (a.m > 0) {
        const hipError_t e = by_length_back(a.n, [&](auto L, auto I) -> hipError_t {
            constexpr int l = decltype(L)::value, i = decltype(I)::value;
            const int rows = l < 64 ? 4 : Row<l>::ROWS;      // parts of a workgroup
            const dim3 grid((a.groups + rows - 1) / rows), block(Row<l>::THREADS);
            if (l == 16 && a.n < 8) {
                if (a.u) EDKM_GO((k_norm_grad<F, 16, 1, true, true, false>), grid, block, a);
                else EDKM_GO((k_norm_grad<F, 16, 1, false, true, false>), grid, block, a);
            } else if (12 * a.m * a.n > INFINITY_CACHE) {
                if (a.u) EDKM_GO((k_norm_grad<F, l, i, true, false, true>), grid, block, a);
                else EDKM_GO((k_norm_grad<F, l, i, false, false, true>), grid, block, a);
            } else {
                if (a.u) EDKM_GO((k_norm_grad<F, l, i, true, false, false>), grid, block, a);
                else EDKM_GO((k_norm_grad<F, l, i, false, false, false>), grid, block, a);
            }
            return hipSuccess;
        });
        if (e != hipSuccess) return e;
    }
    if (a.dw || a.dpost || (a.dgate && !a.gate_rows)) EDKM_GO(k_norm_join<F>, dim3((a.n + 31) / 32, 2), dim3(1024), a);
    return hipSuccess;
}

hipError_t launch_norm(NormArgs a, int fmt, hipStream_t s) { return fmt == FMT_BF16 ? norm_f<FMT_BF16>(a, s) : norm_f<FMT_FP16>(a, s); }
hipError_t launch_norm_backward(NormArgs a, int fmt, hipStream_t s) {
    return fmt == FMT_BF16 ? grad_f<FMT_BF16>(a, s) : grad_f<FMT_FP16>(a, s);
}

}  // namespace edkm
