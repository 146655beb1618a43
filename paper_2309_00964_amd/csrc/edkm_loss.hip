// Softmax cross entropy of a product with a vocabulary, for gfx950 (MI355X): the logits'
// tiles end as their rows' statistics, or as the gradient at the logits, and are never in
// memory themselves.

#include "edkm_loss.h"

#include <algorithm>

namespace edkm {

// ----------------------------------------------------------------------------
// tokens with a target

// One workgroup lists the tokens with a target in order, for a backward those whose loss has a
// gradient; a backward's factors follow, once their largest is known.  What the products
// read has no row of any other token, so whatever those hold (NaN, Inf) reaches no gradient.
constexpr int PICK = 8;      // tokens of a thread at a time

// What a gradient counts for the largest: one that is not finite nothing, so that its token
// alone has a factor that is not finite.  (Without any other the largest is 1.)
__device__ __forceinline__ float size_of(float g) { return __builtin_isfinite(g) ? fabsf(g) : 0.f; }
// In two factors, whose product may be a subnormal number although dx and dw are not.
__device__ __forceinline__ void scales(const PickArgs& a, float top, int count) {
    a.r.alpha[0] = 1.f / 32768.f / (a.reduction == RED_MEAN ? (float)max(count, 1) : 1.f);
    a.r.alpha[1] = top;
}

template <int IDX>
__global__ void __launch_bounds__(1024) k_pick(PickArgs a) {
    __shared__ int waves[2][16];
    __shared__ float tops[16];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int base = 0, turn = 0;
    float top = 0.f;
    for (int64_t i0 = 0; i0 < a.m; i0 += 1024 * PICK, turn ^= 1) {
        const int64_t i = i0 + threadIdx.x * PICK;
        int t[PICK], mine = 0;
        float g[PICK];
#pragma unroll
        for (int e = 0; e < PICK; ++e) {
            t[e] = i + e < a.m ? word_of<IDX>(a.targets, i + e, a.n) : -1;
            g[e] = a.backward && i + e < a.m ? a.dloss[a.reduction == RED_NONE ? i + e : 0] : 1.f;
        }
#pragma unroll
        for (int e = 0; e < PICK; ++e) {
            if (g[e] == 0.f) t[e] = -1;
            mine += t[e] >= 0;
        }
        int run = mine;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int up = __shfl_up(run, o);
            if (lane >= o) run += up;
        }
        if (lane == 63) waves[turn][w] = run;
        __syncthreads();
        int at = base + run - mine;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int c = waves[turn][q];
            at += q < w ? c : 0;
            base += c;
        }
#pragma unroll
        for (int e = 0; e < PICK; ++e) {
            if (i + e >= a.m) break;
            if (a.backward) a.r.slot[i + e] = t[e] >= 0 ? at : -1;
            if (t[e] >= 0) {
                a.r.row[at] = (int)(i + e);
                a.r.word[at] = t[e];
                if (a.backward) {
                    a.r.value[at] = g[e];
                    top = fmaxf(top, size_of(g[e]));
                }
                ++at;
            } else {
                if (a.loss && a.reduction == RED_NONE) a.loss[i + e] = 0.f;
                if (a.lse) a.lse[i + e] = 0.f;
            }
        }
    }
    if (threadIdx.x == 0) a.r.count[0] = base;
    if (!a.backward) return;
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) tops[w] = top;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 16; ++q) top = fmaxf(top, tops[q]);
    if (top == 0.f) top = 1.f;
    for (int i = threadIdx.x; i < base; i += 1024) a.r.value[i] = a.r.value[i] / top * 32768.f;
    if (threadIdx.x == 0) scales(a, top, base);
}

hipError_t launch_pick(const PickArgs& a, int index_type, hipStream_t s) {
    if (index_type == IDX_64) EDKM_GO(k_pick<IDX_64>, dim3(1), dim3(1024), a);
    else EDKM_GO(k_pick<IDX_32>, dim3(1), dim3(1024), a);
    return hipSuccess;
}

// Zeros into a row, by `threads` threads of which this is the t-th.
__device__ __forceinline__ void clear_row(uint16_t* to, int k, int t, int threads) {
    for (int64_t c = t * 8; c < k; c += threads * 8) {
        if (c + 8 <= k) {
            reinterpret_cast<S16x8*>(to + c)->v = s16x8{};
        } else {
            for (int64_t e = c; e < k; ++e) to[e] = 0;
        }
    }
}

// A row to a group of threads: 256 where rows are long.
__global__ void __launch_bounds__(256) k_gather(GatherArgs a, int threads) {
    const int count = *a.r.count;
    const int64_t i = (int64_t)(a.first + blockIdx.x) * (256 / threads) + threadIdx.x / threads;
    if (i >= a.m) return;
    if (i < count && (a.always || count < a.m)) {
        const uint16_t* from = a.x + (int64_t)a.r.row[i] * a.ldx;
        uint16_t* to = a.out + i * a.ldo;
        for (int64_t c = threadIdx.x % threads * 8; c < a.k; c += threads * 8)
            *reinterpret_cast<s16x8*>(to + c) = row8(from + c, a.k - (int)c);
    }
    if (a.zero && a.r.slot[i] < 0) clear_row(a.zero + i * a.ldz, a.k, threadIdx.x % threads, threads);
}

hipError_t launch_gather(GatherArgs a, hipStream_t s) {
    int threads = 8;
    while (threads < 256 && threads * 8 < a.k) threads *= 2;
    const int rows = 256 / threads;
    EDKM_GO_PARTS(k_gather, (uint64_t)((a.m + rows - 1) / rows), 256, a, threads);
    return hipSuccess;
}

// Both for up to 1024 T tokens in one launch: every workgroup makes the list, which the first one
// writes, and then has a share of x's rows, of dx's to clear and of w's to copy, a wave to a row.
// (Losses of 8192 x 1000 x 300 30.5 us, by two launches 34.7, gradients 82 and 90; 1001 x 1003 x 777 38.6, by three 43.8.)
template <int IDX, int T>
__global__ void __launch_bounds__(1024) k_pick_gather(PickArgs a, GatherArgs g, AlignJob w) {
    __shared__ int waves[16], rows[1024 * T];
    __shared__ float tops[16];
    __shared__ unsigned char has[1024 * T];
    const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, i = threadIdx.x * T, m = (int)a.m;
    int t[T], mine = 0;
    float grad[T], top = 0.f;
#pragma unroll
    for (int e = 0; e < T; ++e) {
        t[e] = word_of<IDX>(a.targets, min(i + e, m - 1), a.n);
        grad[e] = 1.f;
    }
    if (a.backward)
#pragma unroll
        for (int e = 0; e < T; ++e) grad[e] = a.dloss[a.reduction == RED_NONE ? min(i + e, m - 1) : 0];
#pragma unroll
    for (int e = 0; e < T; ++e) {
        if (i + e >= m || grad[e] == 0.f) t[e] = -1;
        mine += t[e] >= 0;
        if (t[e] >= 0) top = fmaxf(top, size_of(grad[e]));
    }
    int run = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int up = __shfl_up(run, o);
        if (lane >= o) run += up;
        top = fmaxf(top, __shfl_xor(top, o));
    }
    if (lane == 63) {
        waves[q] = run;
        tops[q] = top;
    }
    __syncthreads();
    int at = run - mine, count = 0;
#pragma unroll
    for (int p = 0; p < 16; ++p) {
        at += p < q ? waves[p] : 0;
        count += waves[p];
        top = fmaxf(top, tops[p]);
    }
    if (top == 0.f) top = 1.f;
    const bool first = blockIdx.x == 0;
    if (first && threadIdx.x == 0) {
        a.r.count[0] = count;
        if (a.backward) scales(a, top, count);
    }
#pragma unroll
    for (int e = 0; e < T; ++e) {
        has[i + e] = t[e] >= 0;
        if (t[e] >= 0) {
            rows[at] = i + e;
            if (first) {
                a.r.row[at] = i + e;
                a.r.word[at] = t[e];
                if (a.backward) a.r.value[at] = grad[e] / top * 32768.f;
            }
            ++at;
        } else if (first && i + e < m) {
            if (a.loss && a.reduction == RED_NONE) a.loss[i + e] = 0.f;
            if (a.lse) a.lse[i + e] = 0.f;
        }
    }
    __syncthreads();
    const bool copy = g.always || count < m;
    const int step = gridDim.x * 16, from = blockIdx.x * 16 + q;
    for (int r = from; r < m; r += step) {
        if (copy && r < count) {
            const uint16_t* x = g.x + (int64_t)rows[r] * g.ldx;
            for (int64_t c = lane * 8; c < g.k; c += 512) *reinterpret_cast<s16x8*>(g.out + r * g.ldo + c) = row8(x + c, g.k - (int)c);
        }
        if (g.zero && !has[r]) clear_row(g.zero + r * g.ldz, g.k, lane, 64);
    }
    // unsigned: w has up to 2^31 - 1025 rows, and the step goes past 2^31
    for (uint32_t r = from; r < (uint32_t)w.rows; r += step)
        for (int64_t c = lane * 8; c < w.cols; c += 512)
            *reinterpret_cast<s16x8*>(w.out + (int64_t)r * ((w.cols + 7) & ~7) + c) = row8(w.m + (int64_t)r * w.ld + c, w.cols - (int)c);
}

template <int T>
static hipError_t pick_gather(const PickArgs& a, const GatherArgs& g, const AlignJob& w, int index_type, hipStream_t s) {
    const dim3 grid((uint32_t)std::min<int64_t>(512, (std::max<int64_t>(a.m, w.rows) + 15) / 16));
    if (index_type == IDX_64) EDKM_GO((k_pick_gather<IDX_64, T>), grid, dim3(1024), a, g, w);
    else EDKM_GO((k_pick_gather<IDX_32, T>), grid, dim3(1024), a, g, w);
    return hipSuccess;
}
hipError_t launch_pick_gather(const PickArgs& a, const GatherArgs& g, const AlignJob& w, int index_type, hipStream_t s) {
    return a.m <= 1024 ? pick_gather<1>(a, g, w, index_type, s) : pick_gather<8>(a, g, w, index_type, s);
}

// ----------------------------------------------------------------------------
// statistics of the blocks of 64 words to losses

// R rows per workgroup: sixteen, or one where there are few tokens.
template <int R>
__global__ void __launch_bounds__(1024) k_loss_end(LossEndArgs a) {
    __shared__ float2 part[16][R];
    const int rows = a.targets ? a.rows : min(a.rows, *a.r.count - a.base);
    const int row = blockIdx.x * R + threadIdx.x % R, q = threadIdx.x / R, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if ((int)blockIdx.x * R >= rows) return;
    const float none = -__builtin_inff();
    float top = none, sum = 0.f;
    auto add = [&](float t, float s) {
        const float m = fmaxf(top, t), from = m == none ? 0.f : m;
        sum = sum * exp_of(top - from) + s * exp_of(t - from);
        top = m;
    };
    constexpr int U = 8, STEP = 1024 / R;
    const int at = min(row, rows - 1);
    for (int b = q; b < a.blocks; b += STEP * U) {
        float2 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = a.stats[(int64_t)min(b + u * STEP, a.blocks - 1) * a.stat_rows + at];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b + u * STEP < a.blocks) add(v[u].x, v[u].y);
    }
#pragma unroll
    for (int o = R; o < 64; o *= 2) {
        const float t = __shfl_xor(top, o), s = __shfl_xor(sum, o);
        add(t, s);
    }
    if (lane < R) part[w][lane] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x >= R || (row >= rows && !a.whole)) return;
    top = none;
    sum = 0.f;
#pragma unroll
    for (int p = 0; p < 16; ++p) add(part[p][lane].x, part[p][lane].y);
    if (a.whole) {
        // the only workgroup: the sum over its rows too
        const bool there = row < rows && word_of(a.targets, a.index_type, row, a.words) >= 0;
        const float l = logf(sum);
        float total = there ? (top - a.r.value[row]) + l : 0.f;
        int count = there;
        if (row < rows && a.lse) a.lse[row] = there ? top + l : 0.f;
#pragma unroll
        for (int o = 1; o < R; o *= 2) {
            total += __shfl_xor(total, o);
            count += __shfl_xor(count, o);
        }
        if (threadIdx.x == 0) a.loss[0] = a.reduction == RED_MEAN ? total / (float)max(count, 1) : total;
        return;
    }
    const bool there = !a.targets || word_of(a.targets, a.index_type, a.base + row, a.words) >= 0;
    const float l = logf(sum), loss = there ? (top - a.r.value[a.base + row]) + l : 0.f;
    const int i = a.targets ? a.base + row : a.r.row[a.base + row];
    if (a.reduction == RED_NONE) a.loss[i] = loss;
    else a.r.value[a.base + row] = loss;
    if (a.lse) a.lse[i] = there ? top + l : 0.f;
}

hipError_t launch_loss_end(const LossEndArgs& a, hipStream_t s) {
    if (a.whole) EDKM_GO(k_loss_end<16>, dim3(1), dim3(1024), a);
    else if (a.rows <= 64) EDKM_GO(k_loss_end<1>, dim3(a.rows), dim3(1024), a);
    else EDKM_GO(k_loss_end<16>, dim3((a.rows + 15) / 16), dim3(1024), a);
    return hipSuccess;
}

__global__ void __launch_bounds__(1024) k_loss_reduce(LossEndArgs a) {
    __shared__ float waves[16];
    int count;
    if (a.targets) {
        // no list: every token's loss is there, 0 for one without a target
        __shared__ int counts[16];
        const bool there = (int)threadIdx.x < a.rows && word_of(a.targets, a.index_type, threadIdx.x, a.words) >= 0;
        const int mine = __popcll(__ballot(there));
        if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = mine;
        __syncthreads();
        count = 0;
        for (int q = 0; q < 16; ++q) count += counts[q];
    } else {
        count = *a.r.count;
    }
    const int there = a.targets ? a.rows : count;
    // many tokens: a thread's long sum keeps what its additions round off
    float sum = 0.f, lost = 0.f;
    for (int i = threadIdx.x; i < there; i += 1024) {
        const float v = a.r.value[i], t = sum + v, z = t - sum;
        lost += (sum - (t - z)) + (v - z);
        sum = t;
    }
    sum += __builtin_isfinite(lost) ? lost : 0.f;
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    sum = 0.f;
    for (int q = 0; q < 16; ++q) sum += waves[q];
    a.loss[0] = a.reduction == RED_MEAN ? sum / (float)max(count, 1) : sum;
}

hipError_t launch_loss_reduce(const LossEndArgs& a, hipStream_t s) {
    EDKM_GO(k_loss_reduce, dim3(1), dim3(1024), a);
    return hipSuccess;
}

// ----------------------------------------------------------------------------
// the products with the vocabulary

// By the time of the launch's rounds over the CUs, in us: a round's steps, one CU's workgroups side
// by side, and what a tile costs beside them (its first loads, its end).  Splitting the depths
// adds a launch and the parts' way to memory and back.  Measured for 256, 128 and 64: 4096 x 4096 x 4096
// 114, 132 and 217; 200 x 32000 x 4096 95, 77 and 120; 1001 x 1003 x 777 32, 19 and 12; 90 x 5000 x 704 20,
// 11 and 7; dw of 64 tokens x 512 and 32000 words 14, 14 and 25; dx of 1536 of 2048 tokens x 2048 over 65536
// words 382 by 256 in five parts, 526 by 128 in two.
LossPlan loss_plan(int64_t rows, int64_t cols, int64_t depth, bool direct) {
    const int64_t steps = std::max<int64_t>(1, (depth + 63) / 64);
    LossPlan best{};
    best.direct = direct;
    double least = 0;
    auto consider = [&](int tile, int64_t most, double alone, double full, double beside) {
        const int64_t t = ((rows + tile - 1) / tile) * ((cols + tile - 1) / tile);
        const int64_t many = t < most ? std::max<int64_t>(1, std::min(most / t, steps / PART_STEPS)) : 1;
        for (const int64_t want : {(int64_t)1, many}) {
            const int64_t each = (steps + want - 1) / want, parts = (steps + each - 1) / each, all = t * parts;
            const double cost = (double)((all + most - 1) / most) * ((double)each * (all <= 256 ? alone : full) + beside) +
                                (parts > 1 ? 4 + (double)all * tile * tile * 8 / 5e6 : 0);
            if (best.tile && cost >= least) continue;
            least = cost;
            best.tile = tile;
            best.splits = (int)parts;
            best.split_steps = (int)each;
            best.groups = parts > 1 ? (int)most : 0;
        }
    };
    consider(128, 512, 0.77, 1.0, 4);
    if (direct) consider(SMALL, 512, 0.3, 0.39, 2.5);
    if (direct) consider(256, 256, 1.6, 1.6, 7);
    return best;
}

size_t loss_part_bytes(int64_t rows, int64_t cols, int64_t depth) {
    size_t most = 0;
    for (const bool direct : {false, true}) {
        const LossPlan q = loss_plan(rows, cols, depth, direct);
        if (q.groups) most = std::max(most, (size_t)q.groups * q.tile * q.tile * 4);
    }
    return most;
}

hipError_t launch_loss_stats(const LossArgs& a, int fmt, const LossPlan& q, hipStream_t s) {
    return fmt == FMT_BF16 ? loss_tiled<FMT_BF16, OP_ROWS, OP_ROWS, LossStats>(a, q, s)
                           : loss_tiled<FMT_FP16, OP_ROWS, OP_ROWS, LossStats>(a, q, s);
}
hipError_t launch_loss_dz(const LossArgs& a, int fmt, const LossPlan& q, hipStream_t s) {
    return fmt == FMT_BF16 ? loss_tiled<FMT_BF16, OP_ROWS, OP_ROWS, LossDz<FMT_BF16>>(a, q, s)
                           : loss_tiled<FMT_FP16, OP_ROWS, OP_ROWS, LossDz<FMT_FP16>>(a, q, s);
}

}  // namespace edkm
