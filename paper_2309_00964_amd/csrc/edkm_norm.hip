// The step from one block to the next, for gfx950 (MI355X): the norm of a block's output,
// its gate and scale, the residual addition and the next block's norm in one pass, and the
// gradients of all of them in another.

#include "edkm_model.h"
#include "edkm_product.h"

#include <algorithm>

namespace edkm {

// L threads share a row, each with I pieces of eight columns.
template <int L>
struct Row {
    static constexpr int THREADS = L < 256 ? 256 : L;
    static constexpr int ROWS = THREADS / L;      // of a workgroup, side by side
    static constexpr int WAVES = L / 64;

    // Sums of a row's K values over its threads.  Sums that follow one another take different
    // places in LDS, so that one barrier each is enough.
    template <int K>
    __device__ __forceinline__ static void sum(float (&v)[K], float (*lds)[16], int place) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int o = 32; o; o >>= 1) v[k] += __shfl_xor(v[k], o);
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
template <int F>
__device__ __forceinline__ void put8(uint16_t* q, const float (&f)[8], int left) {
    s16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (short)to_16<F>(f[j]);
    if (left >= 8) {
        reinterpret_cast<S16x8*>(q)->v = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) q[j] = (uint16_t)v[j];
}

__device__ __forceinline__ float over_root(float sum, const NormArgs& a) {
    return __builtin_amdgcn_rsqf(fmaf(sum, 1.0f / (float)a.n, a.eps));
}

// A row lies in its threads' registers from its loads to its stores; the vectors stay there
// from row to row.  Bound by its bytes: r, u (and a gate's) read, h and y written, once.
template <int F, int L, int I, bool BLOCK>
__global__ void __launch_bounds__(Row<L>::THREADS) k_norm(NormArgs a) {
    typedef Row<L> R;
    __shared__ float lds[6][16];
    const int l = threadIdx.x % L;
    s16x8 w[I], post[I], gate[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = (i * L + l) * 8;
        w[i] = row8(a.w + c, a.n - c);
        if (BLOCK && a.post) post[i] = row8(a.post + c, a.n - c);
        if (BLOCK && a.gate && !a.gate_rows) gate[i] = row8(a.gate + c, a.n - c);
    }
    for (int64_t r = (int64_t)blockIdx.x * R::ROWS + threadIdx.x / L; r < a.m; r += (int64_t)gridDim.x * R::ROWS) {
        float h[I][8];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8;
            floats<F>(row8(a.r + r * a.ldr + c, a.n - c), h[i]);
        }
        if (BLOCK) {
            float b[I][8], ss[1] = {0.f};
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int c = (i * L + l) * 8;
                floats<F>(row8(a.u + r * a.ldu + c, a.n - c), b[i]);
                if (a.gate_rows) gate[i] = row8(a.gate + r * a.ldg + c, a.n - c);
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
// columns' shares of the vectors' gradients in fp32 over its rows; k_norm_join adds the threads'.
template <int F, int L, int I, bool BLOCK>
__global__ void __launch_bounds__(Row<L>::THREADS) k_norm_grad(NormArgs a) {
    typedef Row<L> R;
    __shared__ float lds[9][16];
    const int l = threadIdx.x % L;
    const float per = 1.0f / (float)a.n;
    float sw[I][8] = {}, sp[BLOCK ? I : 1][8] = {}, sg[BLOCK ? I : 1][8] = {};
    const uint32_t group = blockIdx.x * R::ROWS + threadIdx.x / L;
    s16x8 w[I], post[I], gate[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = (i * L + l) * 8;
        w[i] = row8(a.w + c, a.n - c);
        if (BLOCK && a.post) post[i] = row8(a.post + c, a.n - c);
        if (BLOCK && a.gate && !a.gate_rows) gate[i] = row8(a.gate + c, a.n - c);
    }
    for (int64_t r = group; r < a.m; r += a.groups) {
        s16x8 u[I];
        float dy[I][8], d[I][8], h[I][8], su = 1.f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8, left = a.n - c;
            floats<F>(row8(a.r + r * a.ldr + c, left), h[i]);
            floats<F>(a.dy ? row8(a.dy + r * a.lddy + c, left) : s16x8{}, dy[i]);
            floats<F>(a.dh ? row8(a.dh + r * a.lddh + c, left) : s16x8{}, d[i]);
            if (BLOCK) {
                u[i] = row8(a.u + r * a.ldu + c, left);
                if (a.gate_rows) gate[i] = row8(a.gate + r * a.ldg + c, left);
            }
        }
        if (BLOCK) {
            if (a.post) {
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
            }
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = a.gate ? a.scale * to_f32<F>((uint16_t)gate[i][j]) : a.scale;
                    const float p = a.post ? su * to_f32<F>((uint16_t)post[i][j]) : 1.f;
                    h[i][j] = fmaf(g, to_f32<F>((uint16_t)u[i][j]) * p, h[i][j]);
                }
        }
        float s[2] = {0.f, 0.f}, s2[1] = {0.f};
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[0] = fmaf(h[i][j], h[i][j], s[0]);
                s[1] = fmaf(dy[i][j] * to_f32<F>((uint16_t)w[i][j]), h[i][j], s[1]);
            }
        R::sum(s, lds, 1);
        const float sh = over_root(s[0], a), mean = s[1] * sh * per;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int c = (i * L + l) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float hn = h[i][j] * sh;
                d[i][j] = fmaf(sh, fmaf(-hn, mean, dy[i][j] * to_f32<F>((uint16_t)w[i][j])), d[i][j]);
                sw[i][j] = fmaf(dy[i][j], hn, sw[i][j]);
            }
            if (a.dr) put8<F>(a.dr + r * a.lddr + c, d[i], a.n - c);
            if (BLOCK) {
                // h's registers take the gate's gradient from here on, d's the block's
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float un = to_f32<F>((uint16_t)u[i][j]) * su, q = a.scale * d[i][j];
                    const float p = a.post ? to_f32<F>((uint16_t)post[i][j]) : 1.f;
                    const float g = a.gate ? to_f32<F>((uint16_t)gate[i][j]) : 1.f;
                    h[i][j] = q * un * p;
                    sg[i][j] += h[i][j];
                    sp[i][j] = fmaf(q * g, un, sp[i][j]);
                    d[i][j] = q * g * p;
                    s2[0] = fmaf(d[i][j], un, s2[0]);
                }
                if (a.dgate && a.gate_rows) put8<F>(a.dgate + r * a.n + c, h[i], a.n - c);
            }
        }
        if (BLOCK && a.post) R::sum(s2, lds, 2);
        else if (R::WAVES > 1) __syncthreads();      // place 1 is free for the next row
        if (BLOCK && a.du) {
            const float mean2 = s2[0] * per;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int c = (i * L + l) * 8;
                if (a.post)
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[i][j] = su * fmaf(-to_f32<F>((uint16_t)u[i][j]) * su, mean2, d[i][j]);
                put8<F>(a.du + r * a.lddu + c, d[i], a.n - c);
            }
        }
    }
    if (group >= a.groups) return;
    auto keep = [&](int k, const float (&v)[8], int c) {
        float* q = a.part + ((int64_t)group * 3 + k) * a.n + c;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < a.n) q[j] = v[j];
    };
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int c = (i * L + l) * 8;
        if (a.dw) keep(0, sw[i], c);
        if constexpr (BLOCK) {
            if (a.dpost) keep(1, sp[i], c);
            if (a.dgate && !a.gate_rows) keep(2, sg[i], c);
        }
    }
}

// 32 columns of one vector per workgroup, their parts shared by 32 threads each
template <int F>
__global__ void __launch_bounds__(1024) k_norm_join(NormArgs a) {
    __shared__ float red[32][33];
    const int k = blockIdx.y;
    uint16_t* out = k == 0 ? a.dw : k == 1 ? a.dpost : a.gate_rows ? nullptr : a.dgate;
    if (!out) return;
    const int l = threadIdx.x & 31, q = threadIdx.x >> 5, c = blockIdx.x * 32 + l;
    float sum = 0.f;
    if (c < a.n)
#pragma unroll 4
        for (uint32_t i = q; i < a.groups; i += 32) sum += a.part[((int64_t)i * 3 + k) * a.n + c];
    red[q][l] = sum;
    __syncthreads();
    sum = red[l][q];
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor(sum, o, 32);
    const int mine = blockIdx.x * 32 + q;
    if (l == 0 && mine < a.n) out[mine] = to_16<F>(sum);
}

// ----------------------------------------------------------------------------
// launches

// Threads and pieces of a row by its length.
template <class Go>
static hipError_t by_length(int64_t n, Go go) {
    if (n <= 512) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    if (n <= 1024) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
    if (n <= 2048) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    if (n <= 4096) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    if (n <= 8192) return go(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
    return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}
static int row_threads(int64_t n) { return n <= 1024 ? 64 : n <= 4096 ? 256 : n <= 8192 ? 512 : 1024; }

uint32_t norm_groups(int64_t m, int64_t n) {
    const int64_t side = row_threads(n) == 64 ? 4 : 1;
    return (uint32_t)std::min<int64_t>(m, 512 * side);
}

template <int F>
static hipError_t norm_f(const NormArgs& a, hipStream_t s) {
    return by_length(a.n, [&](auto L, auto I) -> hipError_t {
        constexpr int l = decltype(L)::value, i = decltype(I)::value;
        const dim3 grid((uint32_t)std::min<int64_t>((a.m + Row<l>::ROWS - 1) / Row<l>::ROWS, 2048)), block(Row<l>::THREADS);
        if (a.u) EDKM_GO((k_norm<F, l, i, true>), grid, block, a);
        else EDKM_GO((k_norm<F, l, i, false>), grid, block, a);
        return hipSuccess;
    });
}

template <int F>
static hipError_t grad_f(const NormArgs& a, hipStream_t s) {
    if (a.m > 0) {
        const hipError_t e = by_length(a.n, [&](auto L, auto I) -> hipError_t {
            constexpr int l = decltype(L)::value, i = decltype(I)::value;
            const dim3 grid((a.groups + Row<l>::ROWS - 1) / Row<l>::ROWS), block(Row<l>::THREADS);
            if (a.u) EDKM_GO((k_norm_grad<F, l, i, true>), grid, block, a);
            else EDKM_GO((k_norm_grad<F, l, i, false>), grid, block, a);
            return hipSuccess;
        });
        if (e != hipSuccess) return e;
    }
    if (a.dw || a.dpost || (a.dgate && !a.gate_rows)) EDKM_GO(k_norm_join<F>, dim3((a.n + 31) / 32, 3), dim3(1024), a);
    return hipSuccess;
}

hipError_t launch_norm(NormArgs a, int fmt, hipStream_t s) { return fmt == FMT_BF16 ? norm_f<FMT_BF16>(a, s) : norm_f<FMT_FP16>(a, s); }
hipError_t launch_norm_backward(NormArgs a, int fmt, hipStream_t s) {
    return fmt == FMT_BF16 ? grad_f<FMT_BF16>(a, s) : grad_f<FMT_FP16>(a, s);
}

}  // namespace edkm
