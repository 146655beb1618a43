// Products with an epilogue for gfx950 (MI355X): y = act(x W^T + bias) + residual with
// 16-bit weights, the products of its backward pass and the gradient at its activation.

#include "edkm_tiled.h"

#include <algorithm>

namespace edkm {

// ----------------------------------------------------------------------------
// the gradient at the activation

// A thread takes eight columns of every fourth row of the block's; one pass over dy and z
// (bound by its bytes: 6 B per element with an activation, 2 B without) writes dz and sums
// the bias gradient in fp32, unrounded.  dz is rounded to 16 bits because the matrix units take it
// so in both products, as z is kept in 16 bits to hold a layer's tokens at the size of its
// output; dx and dw are 1.45 times as far off for the two as by their own rounding alone (bf16,
// 0.0024 against 0.0017 relative).  PAST: dy and z are read past the caches, for
// matrices that do not fit them: 8192 x 11008 with silu takes 93 us so (5.8 TB/s) and 111
// through them, 4096 x 4096 21.2 and 19.3.  Without activation 8192 x 11008 takes 30 us (6.0 TB/s, from
// the Infinity Cache in part).
template <int F, int ACT, bool PAST>
__global__ void __launch_bounds__(256) k_dz(DzArgs a) {
    __shared__ float red[4][DZ_COLS];
    const int lane = threadIdx.x & 63, q = threadIdx.x >> 6;
    // workgroups go column block by column block through a chunk of rows
    const uint32_t nc = (a.cols + DZ_COLS - 1) / DZ_COLS, cb = (a.first + blockIdx.x) % nc, chunk = (a.first + blockIdx.x) / nc;
    const int c = cb * DZ_COLS + lane * 8, left = a.cols - c;
    const int r0 = chunk * a.per, r1 = min(r0 + a.per, a.rows);
    float sum[8] = {};
    if (left > 0) {
#pragma unroll 2
        for (int r = r0 + q; r < r1; r += 4) {
            const s16x8 d = row8<PAST>(a.dy + (int64_t)r * a.lddy + c, left);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = to_f32<F>((uint16_t)d[j]);
            if (ACT != ACT_NONE) {
                const s16x8 z = row8<PAST>(a.z + (int64_t)r * a.cols + c, left);
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
    const int l = threadIdx.x & 31, q = threadIdx.x >> 5, c = (a.first + blockIdx.x) * 32 + l;
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
    const int mine = (a.first + blockIdx.x) * 32 + q;
    if (l == 0 && mine < a.cols) a.dbias[mine] = to_16<F>(sum);
}

// ----------------------------------------------------------------------------
// launches

template <int F, int OPA, int OPB>
static hipError_t product_ab(const ProductArgs& p, const ProductPlan& q, hipStream_t s) {
    if (q.tile == 256) return tiled<F, OPA, OPB, 256, 2, 4, true>(p, q, s);
    return q.direct ? tiled<F, OPA, OPB, 128, 2, 2, true>(p, q, s) : tiled<F, OPA, OPB, 128, 2, 2, false>(p, q, s);
}

template <int F>
static hipError_t product_f(ProductArgs p, int opa, int opb, float* part, hipStream_t s) {
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

// A tile and a split of the depths.
//
// What bounds a tile is bringing its operands into LDS, whose bytes per product fall with the
// tile's side: a CU takes 1.5 times as long for one tile of 256 as for two of 128 side by
// side, for twice the outputs (95 against 63 us at 4096 depths), and 0.77 as long for a
// single one of 128.  So the tile whose last round costs least: 2560 x 4096 x 4096 takes 96 us
// by tiles of 256 (102 by 128), 1024 x 11008 x 4096 98 (103), but 2048 x 4096 x 4096 99 (73),
// 512 x 11008 x 4096 93 (59) and 4608 x 4096 x 4096 190 (158).  Unaligned operands, whose way
// through registers the larger tile has no room for, take the smaller.
//
// A split costs a launch and its sums' way to memory and back: 3.6 steps' time and 1/26 of
// one for every tile and part, so it is the number of parts that adds up to least.  Measured
// (us by parts): 128 x 4096 x 4096 1: 47, 4: 19.5, 8: 17.4, 16: 20.4; 512 x 4096 x 4096
// 1: 48, 2: 33.0, 3: 29.7, 4: 30.2, 6: 35.8; 1000 x 1336 x 776 1: 12.1, 2: 16.1, 3: 17.5.
static void shape_plan(int64_t rows, int64_t cols, int64_t depth, bool direct, ProductPlan& q) {
    auto tiles = [&](int64_t b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
    const int64_t steps = std::max<int64_t>(1, (depth + 63) / 64), large = tiles(256), t = tiles(128);
    const int64_t large_cost = (large + 255) / 256 * 6, cost = t / 512 * 4 + (t % 512 > 256 ? 4 : t % 512 ? 3 : 0);
    q.direct = direct;
    q.tile = direct && large_cost < cost ? 256 : 128;
    q.splits = 1;
    if (q.tile == SPLIT_TILE) {
        auto time = [&](int64_t s) { return 26 * ((steps + s - 1) / s) + (s > 1 ? 94 + s * t : 0); };
        for (int s = 2; s <= std::min<int64_t>(64, 512 / t); ++s)
            if (time(s) < time(q.splits)) q.splits = s;
    }
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
        return ((uintptr_t)m & 15) == 0 && ld % 8 == 0 && ld <= DIRECT_LD_MOST && (op == OP_DEPTH || p.depth % 8 == 0 || p.padded);
    };
    shape_plan(p.rows, p.cols, p.depth, whole(p.a, p.lda, opa) && (opb == OP_PALETTE || whole(p.b, p.ldb, opb)), q);
    return q;
}

constexpr int64_t INFINITY_CACHE = 256 << 20;
template <int F>
static hipError_t dz_f(DzArgs a, hipStream_t s) {
    const int chunks = (a.rows + a.per - 1) / a.per;
    if (chunks > 0 && (a.dbias || a.act != ACT_NONE)) {
        const uint64_t groups = (uint64_t)((a.cols + DZ_COLS - 1) / DZ_COLS) * chunks;
        if (a.act == ACT_NONE) {
            EDKM_GO_PARTS((k_dz<F, ACT_NONE, false>), groups, 256, a);
        } else if (6 * (int64_t)a.rows * a.cols > INFINITY_CACHE) {
            if (a.act == ACT_RELU) EDKM_GO_PARTS((k_dz<F, ACT_RELU, true>), groups, 256, a);
            else if (a.act == ACT_GELU) EDKM_GO_PARTS((k_dz<F, ACT_GELU, true>), groups, 256, a);
            else EDKM_GO_PARTS((k_dz<F, ACT_SILU, true>), groups, 256, a);
        } else {
            if (a.act == ACT_RELU) EDKM_GO_PARTS((k_dz<F, ACT_RELU, false>), groups, 256, a);
            else if (a.act == ACT_GELU) EDKM_GO_PARTS((k_dz<F, ACT_GELU, false>), groups, 256, a);
            else EDKM_GO_PARTS((k_dz<F, ACT_SILU, false>), groups, 256, a);
        }
    }
    if (a.dbias) EDKM_GO_PARTS(k_dbias<F>, (uint64_t)(a.cols + 31) / 32, 1024, a, chunks);
    return hipSuccess;
}

hipError_t launch_dz(const DzArgs& a, int fmt, hipStream_t s) {
    return fmt == FMT_BF16 ? dz_f<FMT_BF16>(a, s) : dz_f<FMT_FP16>(a, s);
}

}  // namespace edkm
