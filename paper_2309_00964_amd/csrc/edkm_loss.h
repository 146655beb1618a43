// Device code of the cross entropy: what becomes of a product's sums.
#pragma once
#include "edkm_model.h"
#include "edkm_tiled.h"

namespace edkm {

template <int IDX>
__device__ __forceinline__ int word_of(const void* targets, int64_t i, int64_t n) {
    if (IDX == IDX_64) {
        const uint64_t t = static_cast<const uint64_t*>(targets)[i];
        return t < (uint64_t)n ? (int)t : -1;
    }
    const uint32_t t = static_cast<const uint32_t*>(targets)[i];
    return t < (uint64_t)n ? (int)t : -1;
}
__device__ __forceinline__ int word_of(const void* targets, int index_type, int64_t i, int64_t n) {
    return index_type == IDX_64 ? word_of<IDX_64>(targets, i, n) : word_of<IDX_32>(targets, i, n);
}

// What only the device knows: how many tokens have a target.  They are the rows of z and of
// dx, and the depths of dw.
struct LossBegin {
    typedef LossArgs Args;
    __device__ __forceinline__ static bool begin(LossArgs& p) {
        if (p.dynamic == 0) return split(p);
        const int count = *p.rows_of.count;
        if (p.dynamic == 2) {
            p.depth = count;
            if (p.all && count == p.m) {
                p.b = p.all;
                p.ldb = p.ld_all;
            }
            return split(p);
        }
        if (p.all && count == p.m) {
            p.a = p.all;
            p.lda = p.ld_all;
        }
        p.rows = min(p.rows, count - p.base);
        p.a += (int64_t)p.base * p.lda;
        return p.rows > 0 && split(p);
    }
    // as many parts of the depths as the launch has workgroups for, now that the tiles are known
    __device__ __forceinline__ static bool split(LossArgs& p) {
        if (p.groups) {
            const int tiles = ((p.rows + p.tile - 1) / p.tile) * ((p.cols + p.tile - 1) / p.tile), steps = (p.depth + 63) / 64;
            const int parts = max(1, min(p.groups / tiles, steps / PART_STEPS));
            p.split_steps = max(1, (steps + parts - 1) / parts);
            p.splits = max(1, (steps + p.split_steps - 1) / p.split_steps);
            if (p.splits == 1) p.part = nullptr;
        }
        return true;
    }
};

// Of differences of logits: they are formed first, so that e^(z - top) of the largest is 1.  One fma
// with top's product with log2 e would save an operation and be off by that product's rounding: a
// certain token's loss by 4e-5 at logits of 1000, to either side of 0.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// The lanes r, r + 16, r + 32 and r + 48 together, by exchanges of rows of sixteen lanes.
template <class Op>
__device__ __forceinline__ float four_rows(float v, Op op) {
    const uint32_t a = __float_as_uint(v);
    const auto s = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const uint32_t b = __float_as_uint(op(__uint_as_float(s[0]), __uint_as_float(s[1])));
    const auto t = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return op(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

// The largest of a row's 64 logits and the sum of e^(z - largest), and the target's logit.
// A row's logits lie in the four lanes r, r + 16, r + 32 and r + 48.
struct LossStats : LossBegin {
  // sixteen logits of a row in as many lanes
  __device__ __forceinline__ static void row16(const LossArgs& p, int row, int col, float z) {
    const float none = -__builtin_inff();
    if (col == word_of(p.targets, p.index_type, row, p.cols)) p.rows_of.value[row] = z;
    if (col >= p.cols) z = none;
    float top = z;
#pragma unroll
    for (int o = 1; o < 16; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    float sum = exp_of(z - (top == none ? 0.f : top));
#pragma unroll
    for (int o = 1; o < 16; o *= 2) sum += __shfl_xor(sum, o);
    if (col % 16 == 0) p.stats[(int64_t)(col / 16) * p.stat_rows + row] = make_float2(top, sum);
  }
  template <int TR>
  struct End {
    int word[TR];
    __device__ __forceinline__ void init(const LossArgs& p, int lane, int r) {
        // one kind of load to a loop: a choice inside it would wait for one load after the other
        auto row = [&](int i) { return p.base + min(r + i * 16 + (lane & 15), p.rows - 1); };
        if (!p.targets) {
#pragma unroll
            for (int i = 0; i < TR; ++i) word[i] = p.rows_of.word[row(i)];
        } else if (p.index_type == IDX_64) {
#pragma unroll
            for (int i = 0; i < TR; ++i) word[i] = word_of<IDX_64>(p.targets, row(i), p.cols);
        } else {
#pragma unroll
            for (int i = 0; i < TR; ++i) word[i] = word_of<IDX_32>(p.targets, row(i), p.cols);
        }
    }
    __device__ __forceinline__ void block(const LossArgs& p, int i, char*, int lane, int r0, int c0, f32x4 (&acc)[4], int64_t) {
        if (r0 >= p.rows || c0 >= p.cols) return;
        const int row = r0 + (lane & 15), c = c0 + (lane >> 4) * 4;
        const float none = -__builtin_inff();
        // few blocks have a row's target
        const uint32_t t = (uint32_t)(word[i] - c);
        if (__ballot(t < 52)) {
            float z = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t == j * 16u + e) z = acc[j][e];
            if (t < 52 && (t & 15) < 4 && row < p.rows) p.rows_of.value[p.base + row] = z;
        }
        if (c0 + 64 > p.cols)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + j * 16 + e >= p.cols) acc[j][e] = none;
        float top = none;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[j][e]);
        top = four_rows(top, [](float a, float b) { return fmaxf(a, b); });
        const float from = top == none ? 0.f : top;      // all -Inf: the sum is 0, or NaN if one is
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += exp_of(acc[j][e] - from);
        sum = four_rows(sum, [](float a, float b) { return a + b; });
        if (lane < 16 && row < p.rows) p.stats[(int64_t)(c0 / 64) * p.stat_rows + row] = make_float2(top, sum);
    }
  };
};

// Stores a 16 x 64 block as 16-bit values, whole lines at a time; `to` gives the place of the
// lane's first (row lane / 8) and second (eight rows on) row.
// Columns from p.cols on up to `wide` become zeros.
template <int F, class To>
__device__ __forceinline__ void store_block(const LossArgs& p, char* lds, int lane, int r0, int c0, const f32x4 (&acc)[4], int wide, To to) {
#pragma unroll
    for (int j = 0; j < 4; ++j) epi_put(lds, lane, j, acc[j]);
    epi_order();
    const int c = c0 + (lane & 7) * 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = i * 8 + (lane >> 3), q = (lane & 7) * 2;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(lds + r * 256 + ((q ^ r) * 16));
        const f32x4 hi = *reinterpret_cast<const f32x4*>(lds + r * 256 + (((q + 1) ^ r) * 16));
        if (r0 + r >= p.rows || c >= wide) continue;
        const float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        s16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < p.cols ? (short)to_16<F>(f[e]) : (short)0;
        uint16_t* out = to(i) + c;
        if (c + 8 <= wide) {
            reinterpret_cast<S16x8*>(out)->v = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < wide) out[e] = (uint16_t)v[e];
        }
    }
    epi_order();
}

// dz = factor (e^(z - lse) - [word is the target]), rounded to 16 bits because the matrix
// units take it so in both products; the factor is the token's share of 2^15 times the largest
// |dL/dl|, so that fp16 holds probabilities down to 2^-29 (2^-39 with fewer digits).
template <int F>
struct LossDz : LossBegin {
  template <int TR>
  struct End {
    int word[TR];
    float lse[TR], factor[TR];
    __device__ __forceinline__ void init(const LossArgs& p, int lane, int r) {
#pragma unroll
        for (int i = 0; i < TR; ++i) {
            const int row = min(r + i * 16 + (lane & 15), p.rows - 1);
            word[i] = p.rows_of.word[row];
            factor[i] = p.rows_of.value[row];
            lse[i] = p.lse[p.rows_of.row[row]];
        }
    }
    __device__ __forceinline__ void block(const LossArgs& p, int i, char* lds, int lane, int r0, int c0, f32x4 (&acc)[4], int64_t) {
        const int wide = (p.cols + 7) & ~7;
        if (r0 >= p.rows || c0 >= wide) return;
        const uint32_t t = (uint32_t)(word[i] - p.col0 - c0 - (lane >> 4) * 4);
        const bool any = __ballot(t < 52) != 0;      // few blocks have a row's target
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float share = exp_of(acc[j][e] - lse[i]);
                if (any) share -= t == j * 16u + e ? 1.f : 0.f;
                acc[j][e] = factor[i] * share;
            }
        store_block<F>(p, lds, lane, r0, c0, acc, wide, [&](int q) { return p.out + (int64_t)(r0 + (lane >> 3) + q * 8) * p.ldo; });
    }
  };
};

// dx or dw: the sums of one launch, or with those of the launches before, times alpha.
template <int F>
struct LossSum : LossBegin {
  template <int TR>
  struct End {
    int row[TR][2];         // where the lane's two rows of a block go
    float alpha[2];
    __device__ __forceinline__ void init(const LossArgs& p, int lane, int r) {
        alpha[0] = p.rows_of.alpha[0];
        alpha[1] = p.rows_of.alpha[1];
#pragma unroll
        for (int i = 0; i < TR; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q) row[i][q] = min(r + i * 16 + q * 8 + (lane >> 3), p.rows - 1);
        if (p.scatter)
#pragma unroll
            for (int i = 0; i < TR; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) row[i][q] = p.rows_of.row[row[i][q]];
    }
    __device__ __forceinline__ void block(const LossArgs& p, int i, char* lds, int lane, int r0, int c0, f32x4 (&acc)[4], int64_t place) {
        if (r0 >= p.rows || c0 >= p.cols) return;
        float* at = p.accum + place * 1024 + lane * 4;
        if (!p.begins)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] += *reinterpret_cast<const f32x4*>(at + j * 256);
        if (!p.ends) {
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(at + j * 256) = acc[j];
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = acc[j][e] * alpha[0] * alpha[1];
        store_block<F>(p, lds, lane, r0, c0, acc, p.cols, [&](int q) { return p.out + (int64_t)row[i][q] * p.ldo; });
    }
  };
};

// The same product by tiles of 64 x 64, four steps of 64 depths in LDS and three of them on their
// way, for sizes that make too few larger tiles: there a step takes as long as its loads' way
// from memory, which the steps ahead hide, and twice to four times the CUs have a tile.  A wave
// takes 16 rows.  Every wave waits for its own loads of a step and then for the other waves,
// asks for the step three ahead (into the buffer that all have read one step ago) and multiplies.
// 1001 x 1003 x 777 with its statistics takes 12 us so, and 19 by tiles of 128 two steps deep.
constexpr int SMALL_WAVES = 4;
template <int F, int OPA, int OPB, class E>
__global__ void __launch_bounds__(SMALL_WAVES * 64, 2) k_small(LossArgs p) {
    if (!E::begin(p)) return;
    typedef Feed<OPA, SMALL, SMALL_WAVES, true> FA;
    typedef Feed<OPB, SMALL, SMALL_WAVES, true> FB;
    constexpr int BYTES = FA::T::BYTES;
    static_assert(FA::T::PER == 2 && FB::T::PER == 2, "eight loads in two steps");
    static_assert(SMALL_WAVES * EPI_BYTES <= 2 * BYTES, "the epilogue's blocks fit");
    // separate arrays, so that the compiler knows the loads of one buffer apart from the reads of another
    __shared__ __attribute__((aligned(1024))) char a0[BYTES], a1[BYTES], a2[BYTES], a3[BYTES], b0[BYTES], b1[BYTES], b2[BYTES], b3[BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t nx = (p.cols + SMALL - 1) / SMALL, ny = (p.rows + SMALL - 1) / SMALL;
    const uint32_t group = p.first + blockIdx.x, split = group / (nx * ny);
    if (split >= (uint32_t)p.splits) return;
    uint32_t tx, ty;
    tile_of(group % (nx * ny), nx, ny, tx, ty);
    const int r0 = ty * SMALL, c0 = tx * SMALL;
    FA fa;
    FB fb;
    fa.init(p.a, p.lda, r0, p.rows, p.depth, wave, lane);
    fb.init(p.b, p.ldb, c0, p.cols, p.depth, wave, lane);
    typename E::template End<1> end;
    end.init(p, lane, r0 + wave * 16);
    typename FA::T ta;
    typename FB::T tb;
    ta.init(wave * 16, lane);
    tb.init(0, lane);
    f32x4 acc[4] = {};
    const int first = split * p.split_steps, steps = min(first + p.split_steps, (p.depth + 63) / 64);
    // past the last step too, so that as many loads are on their way in every step: they read nothing and write zeros
    auto ask = [&](char* a, char* b, int s) {
        fa.start(a, s * 64);
        fb.start(b, s * 64);
    };
    auto step = [&](const char* a, const char* b, char* an, char* bn, int s) {
        asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");      // its loads of this step, its reads of the last
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        ask(an, bn, s + 3);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const s16x8 va = ta.frag(a, 0, ks);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = mfma16<F>(tb.frag(b, j, ks), va, acc[j]);
        }
    };
    ask(a0, b0, first);
    ask(a1, b1, first + 1);
    ask(a2, b2, first + 2);
    for (int s = first; s < steps; s += 4) {
        step(a0, b0, a3, b3, s);
        if (s + 1 < steps) step(a1, b1, a0, b0, s + 1);
        if (s + 2 < steps) step(a2, b2, a1, b1, s + 2);
        if (s + 3 < steps) step(a3, b3, a2, b2, s + 3);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();       // every load has arrived, and every wave has read
    if (p.part) {
        float* at = p.part + ((int64_t)group * SMALL_WAVES + wave) * 1024 + lane * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(at + j * 256) = acc[j];
        return;
    }
    char* mine = (wave < 2 ? a0 : b0) + (wave & 1) * EPI_BYTES;
    end.block(p, 0, mine, lane, r0 + wave * 16, c0, acc, (int64_t)group * SMALL_WAVES + wave);
}

template <int F, int OPA, int OPB, int B, bool DIRECT, class E>
static hipError_t loss_go(LossArgs p, uint64_t groups, hipStream_t s) {
    if constexpr (B == SMALL) EDKM_GO_PARTS((k_small<F, OPA, OPB, E>), groups, SMALL_WAVES * 64, p);
    else if constexpr (B == 128) EDKM_GO_PARTS((k_tiled<F, OPA, OPB, B, B, 2, 2, DIRECT, 0, E>), groups, 256, p);
    else EDKM_GO_PARTS((k_tiled<F, OPA, OPB, B, B, 2, 4, DIRECT, 0, E>), groups, 512, p);
    return hipSuccess;
}

// With p.groups the launch finds its splits by itself (LossBegin), and there is a join of as
// many blocks as there can be; else every tile takes all depths.
template <int F, int OPA, int OPB, int B, bool DIRECT, class E>
static hipError_t loss_launch(const LossArgs& p, hipStream_t s) {
    constexpr int WM = B == SMALL ? 4 : 2, WN = B == SMALL ? 1 : B == 128 ? 2 : 4;
    const int64_t tiles = ((int64_t)p.cols + B - 1) / B * (((int64_t)p.rows + B - 1) / B);
    const hipError_t e = loss_go<F, OPA, OPB, B, DIRECT, E>(p, p.groups ? p.groups : tiles, s);
    if (e != hipSuccess || !p.groups) return e;
    const dim3 blocks((uint32_t)(tiles * WM * WN * (B / WM / 16)));
    if (p.splits > 8) EDKM_GO((k_join<F, B, B, WM, WN, true, 4, E>), blocks, dim3(256), p, 0);
    else EDKM_GO((k_join<F, B, B, WM, WN, true, 1, E>), blocks, dim3(64), p, 0);
    return hipSuccess;
}

template <int F, int OPA, int OPB, class E>
static hipError_t loss_tiled(const LossArgs& p, const LossPlan& q, hipStream_t s) {
    if (q.tile == 256) return loss_launch<F, OPA, OPB, 256, true, E>(p, s);
    if (q.tile == SMALL) return loss_launch<F, OPA, OPB, SMALL, true, E>(p, s);
    return q.direct ? loss_launch<F, OPA, OPB, 128, true, E>(p, s) : loss_launch<F, OPA, OPB, 128, false, E>(p, s);
}

}  // namespace edkm
