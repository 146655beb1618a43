// C ABI of the layer and optimizer operators: argument checks, workspace layout and
// the launches of each call.  Every check runs on the host before any HIP call.

#include "../../include/edkm.h"
#include "edkm_layer.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <utility>

using namespace edkm;

namespace {

static_assert(EDKM_ACT_NONE == ACT_NONE && EDKM_ACT_RELU == ACT_RELU && EDKM_ACT_GELU == ACT_GELU &&
                  EDKM_ACT_SILU == ACT_SILU, "activations");
static_assert(EDKM_TYPE_FP16 == PT_FP16 && EDKM_TYPE_BF16 == PT_BF16 && EDKM_TYPE_FP32 == PT_FP32, "types");
static_assert(EDKM_STATE_BLOCK == ADAMW_BLOCK, "8-bit state blocks");

constexpr int64_t DIM_MAX = 0x7FFFFFFF - 1024;   // sizes are 32-bit in the kernels, tile ends included

constexpr int64_t MATRIX_MAX = (int64_t)1 << 40;     // elements of a matrix: its tiles are numbered in 32 bits

bool size_ok(int64_t v, int64_t least) { return v >= least && v <= DIM_MAX; }

bool product_ok(int64_t m, int64_t n, int64_t k, int format, int act) {
    return size_ok(m, 0) && size_ok(n, 1) && size_ok(k, 1) && std::max(m, k) <= MATRIX_MAX / n && m <= MATRIX_MAX / k && (format == EDKM_KEYS_FP16 || format == EDKM_KEYS_BF16) &&
           act >= 0 && act < ACT_COUNT;
}

// Leading dimension of a matrix with `rows` rows of `cols`: any for a single row, which
// then gets one that the kernels can work with.
bool ld_ok(int64_t& ld, int64_t rows, int64_t cols) {
    if (rows <= 1) ld = (cols + 7) & ~(int64_t)7;
    return ld >= cols && ld < (int64_t)1 << 40;
}

size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

int64_t dz_chunks(int64_t m, int64_t n) { return (m + dz_rows(m, n) - 1) / dz_rows(m, n); }

int64_t up8(int64_t v) { return (v + 7) & ~(int64_t)7; }

// Rows whose length is no multiple of eight cannot be loaded by 16-byte pieces: a product
// first copies them to rows that can.
size_t aligned_bytes(int64_t rows, int64_t cols) { return cols % 8 ? up256((size_t)rows * up8(cols) * 2) : 0; }

// Workspace of a forward: aligned copies of x and w, then a split product's sums.
struct ForwardWs {
    size_t x, w, split, total;
};
ForwardWs forward_ws(int64_t m, int64_t n, int64_t k) {
    ForwardWs f;
    f.x = 0;
    f.w = f.x + aligned_bytes(m, k);
    f.split = f.w + aligned_bytes(n, k);
    f.total = f.split + up256(product_part_bytes(m, n, k));
    return f;
}

// Workspace of a backward: dz (written with an activation, copied where dy's rows need it),
// the bias gradient's partial sums, aligned copies of x and w, and the split sums of the two
// products in turn.
struct BackwardWs {
    size_t dz, part, x, w, split, total;
};
BackwardWs backward_ws(int64_t m, int64_t n, int64_t k, int act) {
    BackwardWs w;
    w.dz = 0;
    w.part = act == ACT_NONE ? aligned_bytes(m, n) : up256((size_t)m * up8(n) * 2);
    w.x = w.part + up256((size_t)dz_chunks(m, n) * n * 4);
    w.w = w.x + aligned_bytes(m, k);
    w.split = w.w + aligned_bytes(n, k);
    w.total = w.split + up256(std::max(m ? product_part_bytes(m, k, n) : 0, product_part_bytes(n, k, m)));
    return w;
}

// Has a matrix's rows copied to `to`, and points there.
void copy_rows(AlignArgs& a, const uint16_t*& p, int64_t& ld, int64_t rows, int64_t cols, char* to) {
    uint16_t* out = reinterpret_cast<uint16_t*>(to);
    a.job[a.count++] = {p, ld, (int)rows, (int)cols, out};
    p = out;
    ld = up8(cols);
}
// The same, if their length asks for it.
void align_rows(AlignArgs& a, const uint16_t*& p, int64_t& ld, int64_t rows, int64_t cols, char* to) {
    if (cols % 8 && rows > 0) copy_rows(a, p, ld, rows, cols, to);
}

edkm_status ws_ok(const void* ws, size_t have, size_t need) {
    if (need == 0) return EDKM_OK;
    return !ws || have < need || ((uintptr_t)ws & 255u) ? EDKM_ERR_WORKSPACE : EDKM_OK;
}

}  // namespace

extern "C" {

size_t edkm_linear_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (!product_ok(m, n, k, EDKM_KEYS_FP16, EDKM_ACT_NONE) || few_tokens(m, k, false)) return 0;
    return forward_ws(m, n, k).total;
}

edkm_status edkm_linear(int64_t m, int64_t n, int64_t k, int format, int activation, const void* x, int64_t ldx,
                        const void* w, int64_t ldw, const void* bias, const void* residual, int64_t ldr, void* y,
                        int64_t ldy, void* z, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (!product_ok(m, n, k, format, activation) || !w || !ld_ok(ldw, n, k)) return EDKM_ERR_ARG;
    if (m > 0 && (!x || !y)) return EDKM_ERR_ARG;
    if (!ld_ok(ldx, m, k) || !ld_ok(ldy, m, n) || (residual && !ld_ok(ldr, m, n))) return EDKM_ERR_ARG;
    const edkm_status st = ws_ok(ws, ws_bytes, edkm_linear_workspace_bytes(m, n, k));
    if (st != EDKM_OK) return st;
    if (m == 0) return EDKM_OK;
    ProductArgs p{};
    p.a = static_cast<const uint16_t*>(x);
    p.lda = ldx;
    p.b = static_cast<const uint16_t*>(w);
    p.ldb = ldw;
    p.rows = (int32_t)m;
    p.cols = (int32_t)n;
    p.depth = (int32_t)k;
    p.bias = static_cast<const uint16_t*>(bias);
    p.res = static_cast<const uint16_t*>(residual);
    p.ldr = ldr;
    p.out = static_cast<uint16_t*>(y);
    p.ldo = ldy;
    p.z = static_cast<uint16_t*>(z);
    p.act = activation;
    if (few_tokens(m, k, false)) return launch_few(p, format, 0, stream) == hipSuccess ? EDKM_OK : EDKM_ERR_HIP;
    const ForwardWs f = forward_ws(m, n, k);
    char* base = static_cast<char*>(ws);
    p.padded = 1;
    AlignArgs copies{};
    align_rows(copies, p.a, p.lda, m, k, base + f.x);
    align_rows(copies, p.b, p.ldb, n, k, base + f.w);
    if (launch_align_rows(copies, stream) != hipSuccess) return EDKM_ERR_HIP;
    return launch_product(p, format, OP_ROWS, OP_ROWS, reinterpret_cast<float*>(base + f.split), stream) == hipSuccess ? EDKM_OK
                                                                                                                       : EDKM_ERR_HIP;
}

size_t edkm_linear_backward_workspace_bytes(int64_t m, int64_t n, int64_t k, int activation) {
    if (!product_ok(m, n, k, EDKM_KEYS_FP16, activation)) return 0;
    return backward_ws(m, n, k, activation).total;
}

edkm_status edkm_linear_backward(int64_t m, int64_t n, int64_t k, int format, int activation, const void* dy,
                                 int64_t lddy, const void* z, const void* x, int64_t ldx, const void* w, int64_t ldw,
                                 void* dx, int64_t lddx, void* dw, void* dbias, void* ws, size_t ws_bytes,
                                 hipStream_t stream) {
    // without tokens dx is empty, and its pointer may be null
    if (!product_ok(m, n, k, format, activation) || (m > 0 && !dx && !dw && !dbias)) return EDKM_ERR_ARG;
    if (m > 0 && (!dy || (activation != ACT_NONE && !z) || (dw && !x))) return EDKM_ERR_ARG;
    if (dx && (!w || !ld_ok(ldw, n, k) || !ld_ok(lddx, m, k))) return EDKM_ERR_ARG;
    if ((dw && !ld_ok(ldx, m, k)) || !ld_ok(lddy, m, n)) return EDKM_ERR_ARG;
    if (m == 0 && !dw && !dbias) return EDKM_OK;
    const BackwardWs L = backward_ws(m, n, k, activation);
    // without products only dz and the partial sums, which do not depend on k
    const edkm_status st = ws_ok(ws, ws_bytes, dx || dw ? L.total : L.x);
    if (st != EDKM_OK) return st;
    char* base = static_cast<char*>(ws);
    DzArgs d{};
    d.dy = static_cast<const uint16_t*>(dy);
    d.lddy = lddy;
    d.z = static_cast<const uint16_t*>(z);
    d.dz = reinterpret_cast<uint16_t*>(base + L.dz);
    d.part = reinterpret_cast<float*>(base + L.part);
    d.dbias = static_cast<uint16_t*>(dbias);
    d.rows = (int32_t)m;
    d.cols = (int32_t)n;
    d.act = activation;
    d.per = dz_rows(m, n);
    d.lddz = up8(n);
    if (launch_dz(d, format, stream) != hipSuccess) return EDKM_ERR_HIP;
    if (!dx && !dw) return EDKM_OK;
    float* parts = reinterpret_cast<float*>(base + L.split);
    const uint16_t* dz = activation == ACT_NONE ? d.dy : d.dz;
    int64_t lddz = activation == ACT_NONE ? lddy : d.lddz;
    const uint16_t *px = static_cast<const uint16_t*>(x), *pw = static_cast<const uint16_t*>(w);
    AlignArgs copies{};
    if (activation == ACT_NONE) align_rows(copies, dz, lddz, m, n, base + L.dz);
    if (dx && m > 0) align_rows(copies, pw, ldw, n, k, base + L.w);
    if (dw) align_rows(copies, px, ldx, m, k, base + L.x);
    if (launch_align_rows(copies, stream) != hipSuccess) return EDKM_ERR_HIP;
    ProductArgs p{};
    p.a = dz;
    p.lda = lddz;
    p.cols = (int32_t)k;
    p.padded = 1;
    if (dx && m > 0) {
        p.b = pw;
        p.ldb = ldw;
        p.rows = (int32_t)m;
        p.depth = (int32_t)n;
        p.out = static_cast<uint16_t*>(dx);
        p.ldo = lddx;
        if (launch_product(p, format, OP_ROWS, OP_DEPTH, parts, stream) != hipSuccess) return EDKM_ERR_HIP;
    }
    if (dw) {
        p.b = px;
        p.ldb = ldx;
        p.rows = (int32_t)n;
        p.depth = (int32_t)m;
        p.out = static_cast<uint16_t*>(dw);
        p.ldo = k;
        if (launch_product(p, format, OP_DEPTH, OP_DEPTH, parts, stream) != hipSuccess) return EDKM_ERR_HIP;
    }
    return EDKM_OK;
}

// Whether the tiled product decodes the palette itself, once for every tile row: for whole
// pieces of eight indices, where no CU has a second tile.  At 4096 x 4096 and 3 bits it
// takes 21.3 us for 65 tokens, 24.2 for 256, 33.2 for 512 and 58.4 for 1024; decoded first
// by a launch of its own 26.9, 31.2, 38.5 and 59.2.  Past that the decoding that is done over
// and over costs more: 81.0 against 77.8 at 512 x 11008 x 4096, 87.4 against 72.2 for 2048 tokens.
// Tokens that cannot go to LDS directly are copied first (2 to 4 us).
static bool palette_fused(int64_t m, int64_t n, int64_t k, int bits) {
    const int64_t tiles = (m + 127) / 128 * ((n + 127) / 128);
    return tiles <= 256 && k % 8 == 0 && k <= DIRECT_LD_MOST && n * k * bits > 24;
}

size_t edkm_palette_linear_workspace_bytes(int64_t m, int64_t n, int64_t k, int bits) {
    if (!product_ok(m, n, k, EDKM_KEYS_FP16, EDKM_ACT_NONE) || bits < 1 || bits > EDKM_MAX_BITS || few_tokens(m, k, true)) return 0;
    // an aligned copy of x and a split's sums; before them the weights, in rows of whole
    // 16-byte pieces, where they are decoded first
    const size_t parts = up256(product_part_bytes(m, n, k));
    if (palette_fused(m, n, k, bits)) return up256((size_t)m * k * 2) + parts;
    return up256((size_t)n * up8(k) * 2) + aligned_bytes(m, k) + parts;
}

edkm_status edkm_palette_linear(int64_t m, int64_t n, int64_t k, int bits, int format, int activation, const void* x,
                                int64_t ldx, const uint8_t* indices, const float* lut, const void* bias,
                                const void* residual, int64_t ldr, void* y, int64_t ldy, void* z, void* ws,
                                size_t ws_bytes, hipStream_t stream) {
    if (!product_ok(m, n, k, format, activation) || bits < 1 || bits > EDKM_MAX_BITS || !indices || !lut ||
        (uint64_t)n * (uint64_t)k > EDKM_MAX_N)
        return EDKM_ERR_ARG;
    if (m > 0 && (!x || !y)) return EDKM_ERR_ARG;
    if (!ld_ok(ldx, m, k) || !ld_ok(ldy, m, n) || (residual && !ld_ok(ldr, m, n))) return EDKM_ERR_ARG;
    const edkm_status st = ws_ok(ws, ws_bytes, edkm_palette_linear_workspace_bytes(m, n, k, bits));
    if (st != EDKM_OK) return st;
    if (m == 0) return EDKM_OK;
    ProductArgs p{};
    p.a = static_cast<const uint16_t*>(x);
    p.lda = ldx;
    p.idx = indices;
    p.idx_bytes = ((uint64_t)n * (uint64_t)k * (uint64_t)bits + 7) / 8;
    p.lut = lut;
    p.bits = bits;
    p.rows = (int32_t)m;
    p.cols = (int32_t)n;
    p.depth = (int32_t)k;
    p.bias = static_cast<const uint16_t*>(bias);
    p.res = static_cast<const uint16_t*>(residual);
    p.ldr = ldr;
    p.out = static_cast<uint16_t*>(y);
    p.ldo = ldy;
    p.z = static_cast<uint16_t*>(z);
    p.act = activation;
    if (few_tokens(m, k, true)) return launch_few(p, format, bits, stream) == hipSuccess ? EDKM_OK : EDKM_ERR_HIP;
    p.padded = 1;
    AlignArgs copies{};
    if (palette_fused(m, n, k, bits)) {
        if (!product_plan(p, OP_ROWS, OP_PALETTE).direct) copy_rows(copies, p.a, p.lda, m, k, static_cast<char*>(ws));
        float* part = reinterpret_cast<float*>(static_cast<char*>(ws) + up256((size_t)m * k * 2));
        if (launch_align_rows(copies, stream) != hipSuccess) return EDKM_ERR_HIP;
        return launch_tiled_palette(p, format, part, stream) == hipSuccess ? EDKM_OK : EDKM_ERR_HIP;
    }
    char* base = static_cast<char*>(ws);
    uint16_t* w = static_cast<uint16_t*>(ws);
    char* xs = base + up256((size_t)n * up8(k) * 2);
    const hipError_t e = k % 8 ? launch_unpalettize_rows(indices, p.idx_bytes, n, k, bits, format, lut, w, stream)
                               : launch_unpalettize(indices, p.idx_bytes, (uint64_t)n * k, bits, format, lut, w, false, stream);
    p.b = w;
    p.ldb = up8(k);
    align_rows(copies, p.a, p.lda, m, k, xs);
    if (e != hipSuccess || launch_align_rows(copies, stream) != hipSuccess) return EDKM_ERR_HIP;
    return launch_product(p, format, OP_ROWS, OP_ROWS, reinterpret_cast<float*>(xs + aligned_bytes(m, k)), stream) == hipSuccess
               ? EDKM_OK
               : EDKM_ERR_HIP;
}

edkm_status edkm_unpalettize(const uint8_t* indices, uint64_t n, int bits, int format, const float* lut, uint16_t* w_out,
                             hipStream_t stream) {
    if (!indices || !lut || !w_out || n < 1 || n > EDKM_MAX_N || bits < 1 || bits > EDKM_MAX_BITS ||
        (format != EDKM_KEYS_FP16 && format != EDKM_KEYS_BF16))
        return EDKM_ERR_ARG;
    const uint64_t bytes = (n * (uint64_t)bits + 7) / 8;
    return launch_unpalettize(indices, bytes, n, bits, format, lut, w_out, true, stream) == hipSuccess ? EDKM_OK : EDKM_ERR_HIP;
}

edkm_status edkm_adamw_batch(int count, const uint64_t* n, int param_type, int grad_type, int state_bits,
                             void* const* params, float* const* masters, const void* const* grads,
                             void* const* exp_avg, void* const* exp_avg_sq, float* const* m_scales,
                             float* const* v_scales, int32_t* step, const float* lr_dev, double lr, double beta1,
                             double beta2, double eps, double weight_decay, uint32_t seed, hipStream_t stream) {
    if (count < 1 || !n || !params || !grads || !exp_avg || !exp_avg_sq || !step) return EDKM_ERR_ARG;
    if (param_type < PT_FP16 || param_type > PT_FP32 || (grad_type != param_type && grad_type != PT_FP32) ||
        (state_bits != 8 && state_bits != 32) || (state_bits == 8 && (!m_scales || !v_scales)) ||
        (masters && param_type == PT_FP32))
        return EDKM_ERR_ARG;
    if (!(lr_dev || (std::isfinite(lr) && lr >= 0)) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) ||
        !(std::isfinite(eps) && eps >= 0) || !(std::isfinite(weight_decay) && weight_decay >= 0))
        return EDKM_ERR_ARG;
    const size_t pe = param_type == PT_FP32 ? 4 : 2, se = state_bits / 8;
    for (int i = 0; i < count; ++i) {
        if (n[i] > EDKM_MAX_N) return EDKM_ERR_ARG;
        if (n[i] == 0) continue;
        if (!params[i] || !grads[i] || !exp_avg[i] || !exp_avg_sq[i] || (state_bits == 8 && (!m_scales[i] || !v_scales[i])))
            return EDKM_ERR_ARG;
    }
    // Two workgroups must not write the same place: what the tensors of one launch have written.
    // Kinds of arrays go by the address of their first, so that flat buffers come sorted.
    struct Kind {
        const void* const* at;
        size_t size, per;   // bytes for each `per` elements
    };
    Kind kinds[6] = {{params, pe, 1}, {exp_avg, se, 1}, {exp_avg_sq, se, 1}};
    int kinds_n = 3;
    if (masters) kinds[kinds_n++] = {reinterpret_cast<const void* const*>(masters), 4, 1};
    if (state_bits == 8) {
        kinds[kinds_n++] = {reinterpret_cast<const void* const*>(m_scales), 4, ADAMW_BLOCK};
        kinds[kinds_n++] = {reinterpret_cast<const void* const*>(v_scales), 4, ADAMW_BLOCK};
    }
    auto overlap = [&](const int* src, int tensors) {
        typedef std::pair<uintptr_t, uintptr_t> Span;
        Span spans[6 * MAXB];
        int k = 0;
        std::sort(kinds, kinds + kinds_n, [&](const Kind& a, const Kind& b) { return a.at[src[0]] < b.at[src[0]]; });
        for (int q = 0; q < kinds_n; ++q)
            for (int x = 0; x < tensors; ++x) {
                const uintptr_t at = (uintptr_t)kinds[q].at[src[x]];
                if (at) spans[k++] = {at, at + (n[src[x]] + kinds[q].per - 1) / kinds[q].per * kinds[q].size};
            }
        if (!std::is_sorted(spans, spans + k)) std::sort(spans, spans + k);
        for (int x = 1; x < k; ++x)
            if (spans[x].first < spans[x - 1].second) return true;
        return false;
    };
    // by the average launch of the call
    uint64_t total = 0;
    for (int i = 0; i < count; ++i) total += n[i];
    const uint32_t chunk = total / ((count + MAXB - 1) / MAXB) >= ADAMW_MANY ? ADAMW_CHUNK_MANY : ADAMW_CHUNK;
    auto on = [](const void* p, size_t b) { return ((uintptr_t)p & (b - 1)) == 0; };
    AdamwArgs a;
    // all groups are checked before the first launch
    for (int pass = 0; pass < 2; ++pass) {
        for (int i = 0; i < count;) {
            std::memset(&a, 0, sizeof(a));
            a.seed = seed;
            a.step = step;
            a.lr_dev = lr_dev;
            a.lr = lr;
            a.beta1 = beta1;
            a.beta2 = beta2;
            a.eps = eps;
            a.decay = weight_decay;
            a.chunk = chunk;
            a.aligned = 1;
            uint64_t grid = 0;
            int src[MAXB];
            for (; i < count && a.count < MAXB; ++i) {
                if (n[i] == 0) continue;
                const uint64_t wgs = (n[i] + chunk - 1) / chunk;
                if (a.count && grid + wgs > most_groups(256)) break;     // the rest by another launch
                AdamwTensor& T = a.t[a.count];
                T.p = params[i];
                T.master = masters ? masters[i] : nullptr;
                T.g = grads[i];
                T.m = exp_avg[i];
                T.v = exp_avg_sq[i];
                T.m_scale = state_bits == 8 ? m_scales[i] : nullptr;
                T.v_scale = state_bits == 8 ? v_scales[i] : nullptr;
                T.n = n[i];
                // eight elements: 16 bytes of a 16-bit array (fp32 ones are read in two pieces of 16), 8 of a code array
                a.aligned = a.aligned && on(T.p, 16) && on(T.master, 16) && on(T.g, 16) && on(T.m, state_bits == 8 ? 8 : 16) &&
                            on(T.v, state_bits == 8 ? 8 : 16);
                a.wg_begin[a.count] = (uint32_t)grid;
                src[a.count++] = i;
                grid += wgs;
            }
            for (int j = a.count; j < MAXB; ++j) a.wg_begin[j] = 0xFFFFFFFFu;
            if (a.count == 0) continue;
            if (pass == 0) {
                if (overlap(src, a.count)) return EDKM_ERR_ARG;
            } else if (launch_adamw(a, (uint32_t)grid, param_type, grad_type, state_bits, stream) != hipSuccess) {
                return EDKM_ERR_HIP;
            }
        }
    }
    return launch_adamw_tick(step, stream) == hipSuccess ? EDKM_OK : EDKM_ERR_HIP;
}

}  // extern "C"
