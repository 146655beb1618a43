// Embedding for gfx950 (MI355X): rows of a 16-bit or palettized table by token, and the
// table's gradient, summed over tokens that are sorted by their row.

#include "edkm_model.h"
#include "edkm_product.h"

namespace edkm {

// The row of token i, or v for no token.
template <int IDX>
__device__ __forceinline__ uint32_t row_of(const void* ids, int64_t i, uint32_t v) {
    if (IDX == IDX_64) {
        const uint64_t t = static_cast<const uint64_t*>(ids)[i];     // negative: beyond any table
        return t < v ? (uint32_t)t : v;
    }
    const uint32_t t = static_cast<const uint32_t*>(ids)[i];
    return t < v ? t : v;
}

// stores the first `left` of eight values
__device__ __forceinline__ void store8(uint16_t* q, s16x8 v, int left) {
    if (left >= 8) {
        reinterpret_cast<S16x8*>(q)->v = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) q[j] = (uint16_t)v[j];
}

// ----------------------------------------------------------------------------
// lookup

// A thread takes eight columns of four tokens at a time; a workgroup `rows` tokens.  Bound
// by the bytes of the rows read and written.
template <int F, int IDX, int BITS, bool TINY>
__global__ void __launch_bounds__(256) k_embed(EmbedArgs a) {
    constexpr int U = BITS ? 1 : 4;
    Decoder<F> dec;
    if constexpr (BITS != 0) dec.init(a.lut, BITS);
    const uint32_t pieces = (a.d + 7) / 8;
    const bool ragged = a.d % 8 != 0;
    const int64_t i0 = (int64_t)(a.first + blockIdx.x) * a.rows;
    const uint32_t rows = (uint32_t)min((int64_t)a.rows, a.m - i0), total = rows * pieces;
    for (uint32_t l0 = threadIdx.x; l0 < total; l0 += 256 * U) {
        uint32_t r[U], c[U], t[U];
        s16x8 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t l = min(l0 + u * 256, total - 1);
            r[u] = l / pieces;
            c[u] = (l - r[u] * pieces) * 8;
            t[u] = row_of<IDX>(a.ids, i0 + r[u], a.v);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t at = t[u] < a.v ? t[u] : 0;
            if constexpr (BITS != 0) v[u] = dec.eight(load_idx8(a.idx, a.idx_bytes, (uint64_t)at * a.d + c[u], BITS), BITS);
            else v[u] = ask8<TINY>(a.table + (int64_t)at * a.ldt, (int)c[u], (int)a.d);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int left = (int)min(a.d - c[u], 8u);
            if constexpr (BITS == 0) v[u] = had8<TINY>(v[u], left, ragged);
            if (a.scale != 1.f)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[u][j] = (short)to_16<F>(to_f32<F>((uint16_t)v[u][j]) * a.scale);
            if (t[u] >= a.v) v[u] = s16x8{};
            if (l0 + u * 256 < total) store8(a.y + (i0 + r[u]) * a.ldy + c[u], v[u], left);
        }
    }
}

template <int F, int IDX>
static hipError_t embed_fi(EmbedArgs a, int bits, hipStream_t s) {
    const uint32_t pieces = (a.d + 7) / 8;
    a.rows = pieces >= 1024 ? 1 : 1024 / pieces;
    const uint64_t groups = (uint64_t)((a.m + a.rows - 1) / a.rows);
    switch (bits) {
    case 0:
        if (a.d < 8) EDKM_GO_PARTS((k_embed<F, IDX, 0, true>), groups, 256, a);
        else EDKM_GO_PARTS((k_embed<F, IDX, 0, false>), groups, 256, a);
        break;
    case 1: EDKM_GO_PARTS((k_embed<F, IDX, 1, false>), groups, 256, a); break;
    case 2: EDKM_GO_PARTS((k_embed<F, IDX, 2, false>), groups, 256, a); break;
    case 3: EDKM_GO_PARTS((k_embed<F, IDX, 3, false>), groups, 256, a); break;
    default: EDKM_GO_PARTS((k_embed<F, IDX, 4, false>), groups, 256, a); break;
    }
    return hipSuccess;
}

hipError_t launch_embed(EmbedArgs a, int fmt, int index_type, int bits, hipStream_t s) {
    if (fmt == FMT_BF16) return index_type == IDX_64 ? embed_fi<FMT_BF16, IDX_64>(a, bits, s) : embed_fi<FMT_BF16, IDX_32>(a, bits, s);
    return index_type == IDX_64 ? embed_fi<FMT_FP16, IDX_64>(a, bits, s) : embed_fi<FMT_FP16, IDX_32>(a, bits, s);
}

// ----------------------------------------------------------------------------
// tokens by row

// A token's place among the sorted is the number of tokens of lower rows, and of its own row
// before it.  A workgroup counts for 32 tokens, 32 threads to a token, against all tokens
// in LDS: no pass waits for another, and nothing depends on an order of arrival.
template <int IDX>
__global__ void __launch_bounds__(1024) k_rank(SortArgs a) {
    constexpr int T = 1024 / RANK_TOKENS;
    __shared__ __attribute__((aligned(16))) uint32_t all[RANK_MOST];
    __shared__ uint32_t count[T][RANK_TOKENS];
    const uint32_t m4 = (a.m + 3) & ~3u;
#pragma unroll
    for (uint32_t k = 0; k < RANK_MOST / 1024; ++k) {
        const uint32_t j = k * 1024 + threadIdx.x;
        if (j < m4) all[j] = j < a.m ? row_of<IDX>(a.ids, j, a.v) : 0xFFFFFFFFu;
    }
    __syncthreads();
    const uint32_t mine = threadIdx.x & (RANK_TOKENS - 1), q = threadIdx.x / RANK_TOKENS;
    const uint32_t i0 = blockIdx.x * RANK_TOKENS, i = i0 + mine;
    const uint32_t key = i < a.m ? all[i] : 0;
    const uint4* four = reinterpret_cast<const uint4*>(all);
    uint32_t n = 0;
    // tokens before the workgroup's: also those of the same row; after them: lower rows only
#pragma unroll 8
    for (uint32_t j = q; j < i0 / 4; j += T) {
        const uint4 o = four[j];
        n += (o.x <= key) + (o.y <= key) + (o.z <= key) + (o.w <= key);
    }
#pragma unroll 8
    for (uint32_t j = i0 / 4 + RANK_TOKENS / 4 + q; j < m4 / 4; j += T) {
        const uint4 o = four[j];
        n += (o.x < key) + (o.y < key) + (o.z < key) + (o.w < key);
    }
    if (i0 + q < a.m) n += all[i0 + q] < key || (all[i0 + q] == key && q < mine);
    count[q][mine] = n;
    __syncthreads();
    if (threadIdx.x < RANK_TOKENS && i < a.m) {
        uint32_t at = 0;
#pragma unroll
        for (int p = 0; p < T; ++p) at += count[p][mine];
        a.key[at] = key;
        a.pos[at] = i;
    }
}

// A token's row, in the order that the pass before left.
template <int IDX>
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, uint32_t i) {
    return a.key_in ? a.key_in[i] : row_of<IDX>(a.ids, i, a.v);
}
constexpr int KEYS = 4;     // of a thread, loaded side by side

// A pass over one digit of the rows, for more tokens: how many of each digit value a
// workgroup's tokens have ...
template <int IDX>
__global__ void __launch_bounds__(256) k_digits(SortArgs a) {
    __shared__ uint32_t bins[1 << DIGIT_BITS];
    for (uint32_t d = threadIdx.x; d < a.digits; d += 256) bins[d] = 0;
    __syncthreads();
    const uint32_t i0 = blockIdx.x * a.per, i1 = min(i0 + a.per, a.m);
    for (uint32_t i = i0 + threadIdx.x; i < i1; i += 256 * KEYS) {
        uint32_t key[KEYS];
#pragma unroll
        for (int k = 0; k < KEYS; ++k) key[k] = key_of<IDX>(a, min(i + k * 256, i1 - 1));
#pragma unroll
        for (int k = 0; k < KEYS; ++k)
            if (i + k * 256 < i1) atomicAdd(&bins[(key[k] >> a.shift) & (a.digits - 1)], 1u);
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < a.digits; d += 256) a.counts[(uint64_t)blockIdx.x * a.digits + d] = bins[d];
}

// orders a wave's LDS accesses before and after it
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// ... and where they go: behind all lower digits, the same digit in workgroups before this
// one, in waves before this one, and in lanes before this one.  A wave takes its quarter of
// the tokens 64 at a time, in order; the lanes of a digit find each other by a ballot for
// each of its bits.
template <int IDX>
__global__ void __launch_bounds__(256) k_place(SortArgs a) {
    constexpr int MOST = 1 << DIGIT_BITS;
    __shared__ uint32_t next[4][MOST];      // per wave: the next place of a digit
    __shared__ uint32_t scan[4];
    const uint32_t tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const uint32_t share = a.per / 4, i0 = blockIdx.x * a.per + w * share, i1 = min(i0 + share, a.m);
    for (uint32_t d = tid; d < 4 * MOST; d += 256) (&next[0][0])[d] = 0;
    __syncthreads();
    for (uint32_t i = i0 + lane; i < i1; i += 64 * KEYS) {
        uint32_t key[KEYS];
#pragma unroll
        for (int k = 0; k < KEYS; ++k) key[k] = key_of<IDX>(a, min(i + k * 64, i1 - 1));
#pragma unroll
        for (int k = 0; k < KEYS; ++k)
            if (i + k * 64 < i1) atomicAdd(&next[w][(key[k] >> a.shift) & (a.digits - 1)], 1u);
    }
    // a thread sums every 256th digit: all workgroups', and those before this one
    uint32_t below = 0;
    for (uint32_t d0 = 0; d0 < a.digits; d0 += 256) {
        const uint32_t d = d0 + tid, at = min(d, a.digits - 1);
        uint32_t before = 0, total = 0;
        for (uint32_t g = 0; g < a.groups; g += 16) {
            uint32_t c[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) c[k] = a.counts[(uint64_t)min(g + k, a.groups - 1) * a.digits + at];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                total += g + k < a.groups ? c[k] : 0;
                before += g + k < blockIdx.x ? c[k] : 0;
            }
        }
        if (d >= a.digits) total = 0;
        uint32_t run = total;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const uint32_t up = __shfl_up(run, o);
            if ((int)lane >= o) run += up;
        }
        if (lane == 63) scan[w] = run;
        __syncthreads();       // also: the waves' counts are there
        uint32_t start = below + run - total + before;
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
            start += q < w ? scan[q] : 0;
            below += scan[q];
        }
        if (d < a.digits)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t c = next[q][d];
                next[q][d] = start;
                start += c;
            }
        __syncthreads();
    }
    for (uint32_t i = i0; i < i1; i += 64 * KEYS) {
        uint32_t key[KEYS], pos[KEYS];
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            const uint32_t at = min(i + k * 64 + lane, i1 - 1);
            key[k] = key_of<IDX>(a, at);
            pos[k] = a.pos_in ? a.pos_in[at] : at;
        }
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            const bool live = i + k * 64 + lane < i1;
            const uint32_t digit = (key[k] >> a.shift) & (a.digits - 1);
            uint64_t same = __ballot(live);
            for (uint32_t b = 1; b < a.digits; b *= 2) {
                const uint64_t set = __ballot((digit & b) != 0);
                same &= (digit & b) ? set : ~set;
            }
            if (live) {
                const uint32_t at = next[w][digit] + __popcll(same & ((1ull << lane) - 1));
                a.key[at] = key[k];
                a.pos[at] = pos[k];
            }
            wave_order();
            if (live && (same >> lane) == 1) next[w][digit] += __popcll(same);    // the digit's last lane
            wave_order();
        }
    }
}

template <int IDX>
static hipError_t sort_i(SortArgs a, uint32_t* key, uint32_t* pos, uint32_t* spare, hipStream_t s) {
    const SortPlan q = sort_plan(a.m, a.v);
    a.key = key;
    a.pos = pos;
    if (q.passes == 0) {
        EDKM_GO(k_rank<IDX>, dim3((a.m + RANK_TOKENS - 1) / RANK_TOKENS), dim3(1024), a);
        return hipSuccess;
    }
    a.per = q.per;
    a.groups = q.groups;
    a.digits = 1u << q.width;
    // the last pass writes key and pos, those before it in turn
    for (int p = 0; p < q.passes; ++p) {
        const bool last = (q.passes - 1 - p) % 2 == 0;
        a.key = last ? key : spare;
        a.pos = last ? pos : spare + a.m;
        a.shift = p * q.width;
        EDKM_GO(k_digits<IDX>, dim3(a.groups), dim3(256), a);
        EDKM_GO(k_place<IDX>, dim3(a.groups), dim3(256), a);
        a.key_in = a.key;
        a.pos_in = a.pos;
    }
    return hipSuccess;
}

hipError_t launch_sort(const void* ids, int index_type, int64_t m, int64_t v, uint32_t* key, uint32_t* pos, uint32_t* spare,
                       uint32_t* counts, hipStream_t s) {
    SortArgs a{};
    a.ids = ids;
    a.counts = counts;
    a.m = (uint32_t)m;
    a.v = (uint32_t)v;
    return index_type == IDX_64 ? sort_i<IDX_64>(a, key, pos, spare, s) : sort_i<IDX_32>(a, key, pos, spare, s);
}

// ----------------------------------------------------------------------------
// the table's gradient

template <int F>
__device__ __forceinline__ void write_row(const EmbedGradArgs& a, uint32_t t, uint32_t c, const float (&sum)[8]) {
    uint16_t* q = a.dt + (int64_t)t * a.lddt + c;
    const int left = (int)min(a.d - c, 8u);
    s16x8 o;
    if (a.accumulate) {
        const s16x8 old = row8(q, left);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (short)to_16<F>(fmaf(a.scale, sum[j], to_f32<F>((uint16_t)old[j])));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (short)to_16<F>(a.scale * sum[j]);
    }
    store8(q, o, left);
}

// Zeros into n elements from q on, by a workgroup: whole 16-byte places of memory, and the few
// elements before and after them.
__device__ __forceinline__ void clear_span(uint16_t* q, int64_t n, bool past) {
    const int64_t head = min((int64_t)((16 - ((uintptr_t)q & 15)) & 15) / 2, n), body = (n - head) / 8, tail = n - head - body * 8;
    if (threadIdx.x < head) q[threadIdx.x] = 0;
    if (threadIdx.x < tail) q[head + body * 8 + threadIdx.x] = 0;
    s16x8* w = reinterpret_cast<s16x8*>(q + head);
    if (past)
        for (int64_t i = threadIdx.x; i < body; i += 256) __builtin_nontemporal_store(s16x8{}, w + i);
    else
        for (int64_t i = threadIdx.x; i < body; i += 256) w[i] = s16x8{};
}

// The first sorted place whose row is not below t.
__device__ __forceinline__ uint32_t lower(const uint32_t* key, uint32_t m, uint32_t t) {
    uint32_t lo = 0, hi = m;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (key[mid] < t) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// The sorted tokens are cut into chunks of `per`; a thread sums eight columns of a chunk's
// tokens, row by row.  A row whose tokens lie in one chunk is written; what a chunk has of
// others goes to part: place 0 for a row that began in an earlier chunk, place 1 for one
// that begins here and goes on.  Long rows are thereby shared by many threads, and every sum
// has one order.  dy is read past the caches, as it is read once (65536 x 1024 tokens' 36 us, 48
// through them).  Workgroups after those write zeros to the rows of no token, past the caches if the
// table would fill them (8192 tokens of 32000 x 4096: 57 us, 65 through them).
template <int F, bool TINY>
__global__ void __launch_bounds__(256) k_embed_grad(EmbedGradArgs a) {
    const uint32_t group = a.first + blockIdx.x, pieces = (a.d + 7) / 8;
    if (group >= a.chunk_groups) {
        __shared__ uint32_t at[ZERO_MOST + 1];
        const uint32_t t0 = (group - a.chunk_groups) * a.zero_rows, rows = min(a.zero_rows, a.v - t0);
        for (uint32_t r = threadIdx.x; r <= rows; r += 256) at[r] = lower(a.key, a.m, t0 + r);
        __syncthreads();
        if (a.lddt == (int64_t)a.d && a.d < 1024) {
            // short rows without gaps: by the 16-byte places of memory, a thread looking up whose each is
            uint16_t* q = a.dt + (int64_t)t0 * a.d;
            const int n = (int)(rows * a.d), off = (int)(((uintptr_t)q & 15) / 2);
            for (int i = threadIdx.x * 8 - off; i < n; i += 2048) {
                const uint32_t f = (uint32_t)max(i, 0) / a.d, l = (uint32_t)min(i + 7, n - 1) / a.d;
                bool all = i >= 0 && i + 8 <= n;
                for (uint32_t r = f; r <= l; ++r) all = all && at[r] == at[r + 1];
                if (all) {
                    *reinterpret_cast<s16x8*>(q + i) = s16x8{};
                } else {
                    for (int e = max(i, 0); e < min(i + 8, n); ++e)
                        if (at[(uint32_t)e / a.d] == at[(uint32_t)e / a.d + 1]) q[e] = 0;
                }
            }
            return;
        }
        if (a.lddt == (int64_t)a.d) {
            // rows without gaps: all that follow one another at once
            for (uint32_t r = 0; r < rows;) {
                if (at[r] != at[r + 1]) {
                    ++r;
                    continue;
                }
                uint32_t e = r + 1;
                while (e < rows && at[e] == at[e + 1]) ++e;
                clear_span(a.dt + (int64_t)(t0 + r) * a.d, (int64_t)(e - r) * a.d, a.past);
                r = e;
            }
            return;
        }
        uint32_t T = 256;       // threads to a row
        while (T > 8 && T / 2 >= pieces) T /= 2;
        for (uint32_t r = threadIdx.x / T; r < rows; r += 256 / T) {
            if (at[r] != at[r + 1]) continue;
            uint16_t* q = a.dt + (int64_t)(t0 + r) * a.lddt;
            for (uint64_t c = threadIdx.x % T * 8; c < a.d; c += T * 8) store8(q + c, s16x8{}, (int)min(a.d - (uint32_t)c, 8u));
        }
        return;
    }
    const uint64_t id = (uint64_t)group * 256 + threadIdx.x;
    const uint32_t chunk = (uint32_t)(id / pieces), c = (uint32_t)(id - (uint64_t)chunk * pieces) * 8;
    if (chunk >= a.chunks) return;
    const uint32_t j0 = chunk * a.per, j1 = min(j0 + a.per, a.m);
    const int left = (int)min(a.d - c, 8u);
    const uint64_t wide = (uint64_t)pieces * 8;
    const uint32_t before = chunk ? a.key[j0 - 1] : 0xFFFFFFFFu, after = j1 < a.m ? a.key[j1] : 0xFFFFFFFFu;
    uint32_t row = a.key[j0];
    float sum[8] = {};
    auto part = [&](int place) {
        float* q = a.part + ((uint64_t)chunk * 2 + place) * wide + c;
        reinterpret_cast<f32x4*>(q)[0] = f32x4{sum[0], sum[1], sum[2], sum[3]};
        reinterpret_cast<f32x4*>(q)[1] = f32x4{sum[4], sum[5], sum[6], sum[7]};
    };
    constexpr int U = 8;
    const bool ragged = a.d % 8 != 0;
    for (uint32_t j = j0; j < j1 && row < a.v; j += U) {
        s16x8 v[U];
        uint32_t key[U], pos[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t at = min(j + u, j1 - 1);
            key[u] = a.key[at];
            pos[u] = a.pos[at];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = ask8<TINY, true>(a.dy + (int64_t)pos[u] * a.lddy, (int)c, (int)a.d);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j + u >= j1) break;
            if (ragged) v[u] = had8<TINY>(v[u], left, true);
            if (key[u] != row) {
                if (row < a.v) {
                    if (row == before) part(0);
                    else write_row<F>(a, row, c, sum);
                }
                row = key[u];
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += to_f32<F>((uint16_t)v[u][e]);
        }
    }
    if (row >= a.v) return;
    if (row == before) part(0);
    else if (row == after) part(1);
    else write_row<F>(a, row, c, sum);
}

// Adds the parts of the rows that go on past their first chunk: four threads for eight
// columns, each every fourth of the chunks, whose sums are then added in order.  (By sixteen,
// 17 us for 2048 chunks x 1024 where most rows have two parts; by four, 9.)  Rows of fewer than 64
// pieces have up to 32 threads for each, which a workgroup has anyway (131072 tokens of 250 x 64
// added: 32.6 us, by four 61.0).
template <int F>
__global__ void __launch_bounds__(256) k_embed_join(EmbedGradArgs a) {
    __shared__ f32x4 sums[2][256];
    const uint32_t pieces = (a.d + 7) / 8, lanes = 1u << a.lanes, blocks = (pieces + lanes - 1) >> a.lanes, splits = 256 >> a.lanes;
    const uint32_t group = a.first + blockIdx.x, chunk = group / blocks;
    const uint32_t piece = group % blocks * lanes + (threadIdx.x & (lanes - 1)), q = threadIdx.x >> a.lanes;
    const uint32_t j0 = chunk * a.per, row = a.key[j0 + a.per - 1];
    if (row >= a.v || a.key[j0 + a.per] != row || (chunk && a.key[j0 - 1] == row && a.key[j0] == row)) return;
    const uint64_t wide = (uint64_t)pieces * 8;
    const uint32_t c = min(piece, pieces - 1) * 8;
    f32x4 lo = {}, hi = {};
    constexpr int U = 8;
    bool on = true;
    // part 1 of the first chunk, part 0 of those after it
    for (uint32_t k = chunk + q; on && k < a.chunks; k += splits * U) {
        f32x4 l[U], h[U];
        uint32_t key[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t e = min(k + splits * u, a.chunks - 1);
            const float* p = a.part + ((uint64_t)e * 2 + (e == chunk)) * wide + c;
            key[u] = k + splits * u == chunk ? row : k + splits * u < a.chunks ? a.key[e * a.per] : 0xFFFFFFFFu;
            l[u] = reinterpret_cast<const f32x4*>(p)[0];
            h[u] = reinterpret_cast<const f32x4*>(p)[1];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            on = on && key[u] == row;
            if (on) {
                lo += l[u];
                hi += h[u];
            }
        }
    }
    sums[0][threadIdx.x] = lo;
    sums[1][threadIdx.x] = hi;
    __syncthreads();
    if (q || piece >= pieces) return;
#pragma unroll 4
    for (uint32_t p = 1; p < splits; ++p) {
        lo += sums[0][(p << a.lanes) + threadIdx.x];
        hi += sums[1][(p << a.lanes) + threadIdx.x];
    }
    const float sum[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    write_row<F>(a, row, c, sum);
}

template <int F>
static hipError_t grad_f(EmbedGradArgs a, hipStream_t s) {
    const uint64_t threads = (uint64_t)a.chunks * ((a.d + 7) / 8);
    a.zero_rows = max(min((uint32_t)ZERO_VALUES / a.d, (uint32_t)ZERO_MOST), (uint32_t)ZERO_LEAST);
    const uint64_t sums = (threads + 255) / 256, zeros = a.accumulate ? 0 : ((uint64_t)a.v + a.zero_rows - 1) / a.zero_rows;
    a.chunk_groups = (uint32_t)sums;
    a.past = (int64_t)a.v * a.d * 2 > INFINITY_CACHE / 2;
    if (a.d < 8) EDKM_GO_PARTS((k_embed_grad<F, true>), sums + zeros, 256, a);
    else EDKM_GO_PARTS((k_embed_grad<F, false>), sums + zeros, 256, a);
    const uint32_t pieces = (a.d + 7) / 8;
    a.lanes = 6;
    while (a.lanes > 3 && 1u << (a.lanes - 1) >= pieces) --a.lanes;
    if (a.chunks > 1) EDKM_GO_PARTS(k_embed_join<F>, (uint64_t)(a.chunks - 1) * ((pieces + 63) / 64), 256, a);
    return hipSuccess;
}

hipError_t launch_embed_grad(EmbedGradArgs a, int fmt, hipStream_t s) {
    return fmt == FMT_BF16 ? grad_f<FMT_BF16>(a, s) : grad_f<FMT_FP16>(a, s);
}

}  // namespace edkm
