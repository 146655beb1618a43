// C ABI of the operators at a model's ends and between its blocks: argument checks,
// workspace layout and the launches of each call.  Every check runs on the host before any
// HIP call.

#include "edkm_checks.h"
#include "edkm_model.h"

#include <cmath>

using namespace edkm;

namespace {

static_assert(EDKM_INDEX_INT32 == IDX_32 && EDKM_INDEX_INT64 == IDX_64, "index types");
static_assert(LOSS_FEW <= 16, "a workgroup has the rows of a few tokens");
static_assert(EDKM_REDUCE_NONE == RED_NONE && EDKM_REDUCE_SUM == RED_SUM && EDKM_REDUCE_MEAN == RED_MEAN, "reductions");

bool format_ok(int format) { return format == EDKM_KEYS_FP16 || format == EDKM_KEYS_BF16; }
bool index_ok(int type) { return type == EDKM_INDEX_INT32 || type == EDKM_INDEX_INT64; }
edkm_status done(hipError_t e) { return e == hipSuccess ? EDKM_OK : EDKM_ERR_HIP; }

// Its matrices are m x d and v x d.
bool embed_ok(int64_t m, int64_t v, int64_t d, int format, int index_type) {
    return size_ok(m, 0) && size_ok(v, 1) && size_ok(d, 1) && std::max(m, v) <= MATRIX_MAX / d && format_ok(format) && index_ok(index_type);
}

// Workspace of an embedding's backward: the sorted tokens, what their passes need, and the
// chunks' parts of rows that go on.
struct EmbedWs {
    size_t pos, spare, counts, part, total;
    uint32_t per, chunks;
};
EmbedWs embed_ws(int64_t m, int64_t v, int64_t d) {
    EmbedWs w;
    const SortPlan q = sort_plan(m, v);
    w.per = chunk_tokens(m, d);
    w.chunks = (uint32_t)((m + w.per - 1) / w.per);
    w.pos = up256((size_t)m * 4);
    w.spare = w.pos + up256((size_t)m * 4);
    w.counts = w.spare + (q.passes > 1 ? up256((size_t)m * 8) : 0);
    w.part = w.counts + (q.passes ? up256(((size_t)q.groups << q.width) * 4) : 0);
    w.total = w.part + (w.chunks > 1 ? up256((size_t)w.chunks * 2 * up8(d) * 4) : 0);
    return w;
}

bool norm_ok(int64_t m, int64_t n, int format, float scale, float eps) {
    return size_ok(m, 0) && n >= 1 && n <= EDKM_NORM_MAX && format_ok(format) && std::isfinite(scale) && std::isnormal(eps) && eps > 0;
}

// Where a loss's workspace has its lists of tokens.
struct RowsWs {
    size_t row, word, slot, value, x, total;
};
RowsWs rows_ws(int64_t m, int64_t k) {
    RowsWs w;
    const size_t list = up256((size_t)m * 4);
    w.row = 256;
    w.word = w.row + list;
    w.slot = w.word + list;
    w.value = w.slot + list;
    w.x = w.value + list;
    w.total = w.x + up256((size_t)m * up8(k) * 2);
    return w;
}
LossRows rows_at(char* base, const RowsWs& w) {
    LossRows r;
    r.count = reinterpret_cast<int32_t*>(base);
    r.alpha = reinterpret_cast<float*>(base + 128);
    r.row = reinterpret_cast<int32_t*>(base + w.row);
    r.word = reinterpret_cast<int32_t*>(base + w.word);
    r.slot = reinterpret_cast<int32_t*>(base + w.slot);
    r.value = reinterpret_cast<float*>(base + w.value);
    return r;
}

struct LossWs {
    RowsWs rows;
    size_t w, stats, split, total;
};
LossWs loss_ws(int64_t m, int64_t n, int64_t k) {
    LossWs L;
    L.rows = rows_ws(m, k);
    L.w = L.rows.total;
    L.stats = L.w + aligned_bytes(n, k);
    const int64_t rows = loss_rows(m, n);
    L.split = L.stats + up256((size_t)(loss_few(m, k) ? (n + 15) / 16 : (n + 63) / 64) * rows * 8);
    size_t parts = 0;
    if (m > 0) {
        parts = loss_part_bytes(rows, n, k);
        if (m % rows) parts = std::max(parts, loss_part_bytes(m % rows, n, k));
    }
    L.total = L.split + up256(parts);
    return L;
}

struct LossBackWs {
    RowsWs rows;
    size_t w, dz, accum, split, total;
    int64_t piece;
};
LossBackWs loss_back_ws(int64_t m, int64_t n, int64_t k) {
    LossBackWs L;
    L.piece = loss_piece(m, n);
    const int64_t last = n % L.piece;
    L.rows = rows_ws(m, k);
    L.w = L.rows.total;
    L.dz = L.w + aligned_bytes(n, k);
    L.accum = L.dz + up256((size_t)m * up8(L.piece) * 2);
    // tiles of either size
    L.split = L.accum + (L.piece < n ? up256((size_t)((m + 255) / 256 * 256) * ((k + 255) / 256 * 256) * 4) : 0);
    size_t parts = loss_part_bytes(L.piece, k, m);
    if (last) parts = std::max(parts, loss_part_bytes(last, k, m));
    if (m > 0) {
        parts = std::max(parts, loss_part_bytes(m, L.piece, k));
        parts = std::max(parts, loss_part_bytes(m, k, L.piece));
        if (last) parts = std::max(parts, loss_part_bytes(m, last, k));
    }
    L.total = L.split + up256(parts);
    return L;
}

bool loss_ok(int64_t m, int64_t n, int64_t k, int format, int index_type, int reduction) {
    return product_ok(m, n, k, format, ACT_NONE) && index_ok(index_type) && reduction >= 0 && reduction < RED_COUNT;
}

// Rows that a product can take as they are.
bool whole(const void* p, int64_t ld, int64_t k) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && ld <= DIRECT_LD_MOST && k % 8 == 0;
}

void set_plan(LossArgs& p, const LossPlan& q, float* parts) {
    p.split_steps = q.split_steps;
    p.splits = q.groups ? q.splits : 1;
    p.groups = q.groups;
    p.tile = q.tile;
    p.part = q.groups ? parts : nullptr;
}
LossPlan planned(LossArgs& p, int opa, int opb, float* parts) {
    const LossPlan q = loss_plan(p.rows, p.cols, p.depth, product_plan(p, opa, opb).direct);
    set_plan(p, q, parts);
    return q;
}

// The launches that a loss's forward and backward begin with: the list of tokens, their rows
// of x, and w's rows where they have to be copied.
hipError_t begin_loss(const PickArgs& pick, int index_type, const uint16_t* x, int64_t ldx, int64_t k, uint16_t* to, uint16_t* zero,
                      int64_t ldz, const AlignArgs& copies, hipStream_t s) {
    GatherArgs g{};
    g.r = pick.r;
    g.x = x;
    g.ldx = ldx;
    g.out = to;
    g.ldo = up8(k);
    g.m = pick.m;
    g.k = (int)k;
    g.always = !whole(x, ldx, k);
    g.zero = zero;
    g.ldz = ldz;
    if (pick.m > 0 && pick.m <= ONE_LIST) return launch_pick_gather(pick, g, copies.count ? copies.job[0] : AlignJob{}, index_type, s);
    hipError_t e = launch_pick(pick, index_type, s);
    if (e == hipSuccess && pick.m > 0) e = launch_gather(g, s);
    return e == hipSuccess ? launch_align_rows(copies, s) : e;
}

}  // namespace

extern "C" {

edkm_status edkm_embedding(int64_t m, int64_t v, int64_t d, int format, int index_type, const void* ids, const void* table, int64_t ldt,
                           float scale, void* y, int64_t ldy, hipStream_t stream) {
    if (!embed_ok(m, v, d, format, index_type) || !table || !ld_ok(ldt, v, d) || !ld_ok(ldy, m, d) || !std::isfinite(scale)) return EDKM_ERR_ARG;
    if (m > 0 && (!ids || !y)) return EDKM_ERR_ARG;
    if (m == 0) return EDKM_OK;
    EmbedArgs a{};
    a.ids = ids;
    a.table = static_cast<const uint16_t*>(table);
    a.ldt = ldt;
    a.y = static_cast<uint16_t*>(y);
    a.ldy = ldy;
    a.m = m;
    a.v = (uint32_t)v;
    a.d = (uint32_t)d;
    a.scale = scale;
    return done(launch_embed(a, format, index_type, 0, stream));
}

edkm_status edkm_palette_embedding(int64_t m, int64_t v, int64_t d, int bits, int format, int index_type, const void* ids,
                                   const uint8_t* indices, const float* lut, float scale, void* y, int64_t ldy, hipStream_t stream) {
    if (!embed_ok(m, v, d, format, index_type) || bits < 1 || bits > EDKM_MAX_BITS || !indices || !lut || !ld_ok(ldy, m, d) ||
        !std::isfinite(scale) || (uint64_t)v * (uint64_t)d > EDKM_MAX_N)
        return EDKM_ERR_ARG;
    if (m > 0 && (!ids || !y)) return EDKM_ERR_ARG;
    if (m == 0) return EDKM_OK;
    EmbedArgs a{};
    a.ids = ids;
    a.idx = indices;
    a.lut = lut;
    a.idx_bytes = ((uint64_t)v * (uint64_t)d * (uint64_t)bits + 7) / 8;
    a.y = static_cast<uint16_t*>(y);
    a.ldy = ldy;
    a.m = m;
    a.v = (uint32_t)v;
    a.d = (uint32_t)d;
    a.scale = scale;
    return done(launch_embed(a, format, index_type, bits, stream));
}

size_t edkm_embedding_backward_workspace_bytes(int64_t m, int64_t v, int64_t d) {
    if (!embed_ok(m, v, d, EDKM_KEYS_FP16, EDKM_INDEX_INT32) || m == 0) return 0;
    return embed_ws(m, v, d).total;
}

edkm_status edkm_embedding_backward(int64_t m, int64_t v, int64_t d, int format, int index_type, const void* ids, const void* dy,
                                    int64_t lddy, float scale, int accumulate, void* dtable, int64_t lddt, void* ws, size_t ws_bytes,
                                    hipStream_t stream) {
    if (!embed_ok(m, v, d, format, index_type) || !dtable || !ld_ok(lddt, v, d) || !ld_ok(lddy, m, d) || !std::isfinite(scale))
        return EDKM_ERR_ARG;
    if (m > 0 && (!ids || !dy)) return EDKM_ERR_ARG;
    const edkm_status st = ws_ok(ws, ws_bytes, edkm_embedding_backward_workspace_bytes(m, v, d));
    if (st != EDKM_OK) return st;
    if (m == 0 && accumulate) return EDKM_OK;
    EmbedGradArgs a{};
    a.dy = static_cast<const uint16_t*>(dy);
    a.lddy = lddy;
    a.dt = static_cast<uint16_t*>(dtable);
    a.lddt = lddt;
    a.m = (uint32_t)m;
    a.v = (uint32_t)v;
    a.d = (uint32_t)d;
    a.scale = scale;
    a.accumulate = accumulate != 0;
    if (m > 0) {
        const EmbedWs w = embed_ws(m, v, d);
        char* base = static_cast<char*>(ws);
        uint32_t *key = reinterpret_cast<uint32_t*>(base), *pos = reinterpret_cast<uint32_t*>(base + w.pos);
        if (launch_sort(ids, index_type, m, v, key, pos, reinterpret_cast<uint32_t*>(base + w.spare),
                        reinterpret_cast<uint32_t*>(base + w.counts), stream) != hipSuccess)
            return EDKM_ERR_HIP;
        a.key = key;
        a.pos = pos;
        a.part = reinterpret_cast<float*>(base + w.part);
        a.per = w.per;
        a.chunks = w.chunks;
    }
    return done(launch_embed_grad(a, format, stream));
}

edkm_status edkm_residual_norm(int64_t m, int64_t n, int format, const void* r, int64_t ldr, const void* u, int64_t ldu, const void* w,
                               const void* post, const void* gate, int64_t ldg, int gate_rows, float scale, float eps, void* h, int64_t ldh,
                               void* y, int64_t ldy, hipStream_t stream) {
    if (!norm_ok(m, n, format, scale, eps) || !w || !ld_ok(ldr, m, n) || !ld_ok(ldy, m, n) || (m > 0 && (!r || !y))) return EDKM_ERR_ARG;
    const bool rows = gate && gate_rows;
    if ((post || gate || h) && !u && m > 0) return EDKM_ERR_ARG;
    if (u && ((m > 0 && !h) || !ld_ok(ldu, m, n) || !ld_ok(ldh, m, n) || (rows && !ld_ok(ldg, m, n)))) return EDKM_ERR_ARG;
    if (m == 0) return EDKM_OK;
    NormArgs a{};
    a.r = static_cast<const uint16_t*>(r);
    a.u = static_cast<const uint16_t*>(u);
    a.w = static_cast<const uint16_t*>(w);
    a.post = static_cast<const uint16_t*>(post);
    a.gate = static_cast<const uint16_t*>(gate);
    a.ldr = ldr;
    a.ldu = ldu;
    a.ldg = ldg;
    a.gate_rows = rows;
    a.scale = scale;
    a.eps = eps;
    a.h = static_cast<uint16_t*>(h);
    a.y = static_cast<uint16_t*>(y);
    a.ldh = ldh;
    a.ldy = ldy;
    a.m = m;
    a.n = (int)n;
    return done(launch_norm(a, format, stream));
}

size_t edkm_residual_norm_backward_workspace_bytes(int64_t m, int64_t n) {
    if (!norm_ok(m, n, EDKM_KEYS_FP16, 1.f, 1.f) || m == 0) return 0;
    return up256((size_t)norm_groups(m, n) * 2 * n * 4);
}

edkm_status edkm_residual_norm_backward(int64_t m, int64_t n, int format, const void* dy, int64_t lddy, const void* dh, int64_t lddh,
                                        const void* r, int64_t ldr, const void* u, int64_t ldu, const void* w, const void* post,
                                        const void* gate, int64_t ldg, int gate_rows, float scale, float eps, void* dr, int64_t lddr,
                                        void* du, int64_t lddu, void* dw, void* dpost, void* dgate, void* ws, size_t ws_bytes,
                                        hipStream_t stream) {
    if (!norm_ok(m, n, format, scale, eps) || !w || (m > 0 && !r)) return EDKM_ERR_ARG;
    const bool rows = gate && gate_rows;
    if (m > 0 && !u && (post || gate || du)) return EDKM_ERR_ARG;
    if ((dpost && !post) || (dgate && !gate) || (m > 0 && !dr && !du && !dw && !dpost && !dgate)) return EDKM_ERR_ARG;
    if (!ld_ok(ldr, m, n) || (dy && !ld_ok(lddy, m, n)) || (dh && !ld_ok(lddh, m, n)) || (dr && !ld_ok(lddr, m, n)) ||
        (u && !ld_ok(ldu, m, n)) || (du && !ld_ok(lddu, m, n)) || (rows && !ld_ok(ldg, m, n)))
        return EDKM_ERR_ARG;
    const edkm_status st = ws_ok(ws, ws_bytes, edkm_residual_norm_backward_workspace_bytes(m, n));
    if (st != EDKM_OK) return st;
    NormArgs a{};
    a.u = static_cast<const uint16_t*>(u);
    a.w = static_cast<const uint16_t*>(w);
    a.post = static_cast<const uint16_t*>(post);
    a.gate = static_cast<const uint16_t*>(gate);
    a.ldu = ldu;
    a.ldg = ldg;
    a.gate_rows = rows;
    a.scale = scale;
    a.eps = eps;
    a.r = static_cast<const uint16_t*>(r);
    a.ldr = ldr;
    a.m = m;
    a.n = (int)n;
    a.dy = static_cast<const uint16_t*>(dy);
    a.dh = static_cast<const uint16_t*>(dh);
    a.lddy = lddy;
    a.lddh = lddh;
    a.dr = static_cast<uint16_t*>(dr);
    a.du = static_cast<uint16_t*>(du);
    a.dw = static_cast<uint16_t*>(dw);
    a.dpost = static_cast<uint16_t*>(dpost);
    a.dgate = static_cast<uint16_t*>(dgate);
    a.lddr = lddr;
    a.lddu = lddu;
    a.part = static_cast<float*>(ws);
    a.groups = m > 0 ? norm_groups(m, n) : 0;
    return done(launch_norm_backward(a, format, stream));
}

size_t edkm_linear_cross_entropy_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (!loss_ok(m, n, k, EDKM_KEYS_FP16, EDKM_INDEX_INT32, EDKM_REDUCE_NONE)) return 0;
    return loss_ws(m, n, k).total;
}

edkm_status edkm_linear_cross_entropy(int64_t m, int64_t n, int64_t k, int format, int index_type, int reduction, const void* x, int64_t ldx,
                                      const void* w, int64_t ldw, const void* targets, float* loss, float* lse, void* ws, size_t ws_bytes,
                                      hipStream_t stream) {
    if (!loss_ok(m, n, k, format, index_type, reduction) || !w || !ld_ok(ldw, n, k) || !ld_ok(ldx, m, k)) return EDKM_ERR_ARG;
    if (m > 0 && (!x || !targets)) return EDKM_ERR_ARG;
    if (!loss && (m > 0 || reduction != RED_NONE)) return EDKM_ERR_ARG;
    const edkm_status st = ws_ok(ws, ws_bytes, edkm_linear_cross_entropy_workspace_bytes(m, n, k));
    if (st != EDKM_OK) return st;
    if (m == 0 && reduction == RED_NONE) return EDKM_OK;
    const LossWs L = loss_ws(m, n, k);
    char* base = static_cast<char*>(ws);
    const uint16_t *px = static_cast<const uint16_t*>(x), *pw = static_cast<const uint16_t*>(w);
    PickArgs pick{};
    pick.targets = targets;
    pick.m = m;
    pick.n = n;
    pick.reduction = reduction;
    pick.r = rows_at(base, L.rows);
    pick.loss = loss;
    pick.lse = lse;
    uint16_t* xs = reinterpret_cast<uint16_t*>(base + L.rows.x);
    AlignArgs copies{};
    const bool list = m > LIST_LEAST || m == 0, few = loss_few(m, k);
    if (m > 0 && !few) align_rows(copies, pw, ldw, n, k, base + L.w);
    if (list) {
        if (begin_loss(pick, index_type, px, ldx, k, xs, nullptr, 0, copies, stream) != hipSuccess) return EDKM_ERR_HIP;
    } else {
        if (!few && !whole(px, ldx, k)) copy_rows(copies, px, ldx, m, k, reinterpret_cast<char*>(xs));
        if (launch_align_rows(copies, stream) != hipSuccess) return EDKM_ERR_HIP;
    }
    const int64_t most = loss_rows(m, n);
    LossEndArgs end{};
    end.r = pick.r;
    end.stats = reinterpret_cast<float2*>(base + L.stats);
    end.blocks = (int32_t)(few ? (n + 15) / 16 : (n + 63) / 64);
    end.reduction = reduction;
    end.loss = loss;
    end.lse = lse;
    end.targets = list ? nullptr : targets;
    end.index_type = index_type;
    end.words = n;
    end.whole = few && reduction != RED_NONE;
    for (int64_t at = 0; at < m; at += most) {
        const int64_t rows = std::min(most, m - at);
        LossArgs p{};
        p.a = list ? xs : px;
        p.lda = list ? up8(k) : ldx;
        p.b = pw;
        p.ldb = ldw;
        p.rows = (int32_t)rows;
        p.cols = (int32_t)n;
        p.depth = (int32_t)k;
        p.padded = 1;
        p.rows_of = pick.r;
        p.m = (int32_t)m;
        p.targets = end.targets;
        p.index_type = index_type;
        p.stats = reinterpret_cast<float2*>(base + L.stats);
        p.stat_rows = (int32_t)rows;
        if (few) {
            if (launch_few_loss(p, format, stream) != hipSuccess) return EDKM_ERR_HIP;
        } else {
            const LossPlan q = planned(p, OP_ROWS, OP_ROWS, reinterpret_cast<float*>(base + L.split));
            if (list) {
                p.all = whole(x, ldx, k) ? px : nullptr;
                p.ld_all = ldx;
                p.dynamic = 1;
            } else {
                p.a += at * p.lda;
            }
            p.base = (int32_t)at;
            if (launch_loss_stats(p, format, q, stream) != hipSuccess) return EDKM_ERR_HIP;
        }
        end.stat_rows = (int32_t)rows;
        end.base = (int32_t)at;
        end.rows = (int32_t)rows;
        if (launch_loss_end(end, stream) != hipSuccess) return EDKM_ERR_HIP;
    }
    end.rows = (int32_t)m;
    return reduction == RED_NONE || end.whole ? EDKM_OK : done(launch_loss_reduce(end, stream));
}

size_t edkm_linear_cross_entropy_backward_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (!loss_ok(m, n, k, EDKM_KEYS_FP16, EDKM_INDEX_INT32, EDKM_REDUCE_NONE)) return 0;
    return loss_back_ws(m, n, k).total;
}

edkm_status edkm_linear_cross_entropy_backward(int64_t m, int64_t n, int64_t k, int format, int index_type, int reduction, const float* dloss,
                                               const void* x, int64_t ldx, const void* w, int64_t ldw, const void* targets, const float* lse,
                                               void* dx, int64_t lddx, void* dw, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (!loss_ok(m, n, k, format, index_type, reduction) || !w || !ld_ok(ldw, n, k) || !ld_ok(ldx, m, k) || (dx && !ld_ok(lddx, m, k)))
        return EDKM_ERR_ARG;
    if (m > 0 && (!x || !targets || !lse || !dloss || (!dx && !dw))) return EDKM_ERR_ARG;
    if (m == 0 && !dw) return EDKM_OK;
    const edkm_status st = ws_ok(ws, ws_bytes, edkm_linear_cross_entropy_backward_workspace_bytes(m, n, k));
    if (st != EDKM_OK) return st;
    const LossBackWs L = loss_back_ws(m, n, k);
    char* base = static_cast<char*>(ws);
    const uint16_t *px = static_cast<const uint16_t*>(x), *pw = static_cast<const uint16_t*>(w);
    PickArgs pick{};
    pick.targets = targets;
    pick.m = m;
    pick.n = n;
    pick.reduction = reduction;
    pick.r = rows_at(base, L.rows);
    pick.dloss = dloss;
    pick.backward = 1;
    uint16_t *xs = reinterpret_cast<uint16_t*>(base + L.rows.x), *dz = reinterpret_cast<uint16_t*>(base + L.dz);
    AlignArgs copies{};
    if (m > 0) align_rows(copies, pw, ldw, n, k, base + L.w);
    if (begin_loss(pick, index_type, px, ldx, k, xs, m > 0 ? static_cast<uint16_t*>(dx) : nullptr, lddx, copies, stream) != hipSuccess)
        return EDKM_ERR_HIP;
    float* parts = reinterpret_cast<float*>(base + L.split);
    const uint16_t* all = m > 0 && whole(x, ldx, k) ? px : nullptr;
    LossPlan qx{};
    for (int64_t c0 = 0; c0 < n; c0 += L.piece) {
        const int64_t words = std::min(L.piece, n - c0), ldz = up8(L.piece);
        LossArgs p{};
        p.rows_of = pick.r;
        p.m = (int32_t)m;
        p.padded = 1;
        if (m > 0) {
            p.a = xs;
            p.lda = up8(k);
            p.all = all;
            p.ld_all = ldx;
            p.b = pw + c0 * ldw;
            p.ldb = ldw;
            p.rows = (int32_t)m;
            p.cols = (int32_t)words;
            p.depth = (int32_t)k;
            p.dynamic = 1;
            p.col0 = (int32_t)c0;
            p.lse = lse;
            p.out = dz;
            p.ldo = ldz;
            const LossPlan q = planned(p, OP_ROWS, OP_ROWS, parts);
            if (launch_loss_dz(p, format, q, stream) != hipSuccess) return EDKM_ERR_HIP;
        }
        p.a = dz;
        p.lda = ldz;
        p.all = nullptr;
        if (dx && m > 0) {
            p.cols = (int32_t)k;
            p.depth = (int32_t)words;
            // the same for every piece, whose sums are added tile by tile
            if (c0 == 0) qx = planned(p, OP_ROWS, OP_DEPTH, parts);
            else set_plan(p, qx, parts);
            p.accum = reinterpret_cast<float*>(base + L.accum);
            p.begins = c0 == 0;
            p.ends = c0 + words == n;
            p.scatter = 1;
            p.out = static_cast<uint16_t*>(dx);
            p.ldo = lddx;
            if (launch_loss_sum(p, format, OP_ROWS, qx, stream) != hipSuccess) return EDKM_ERR_HIP;
        }
        if (dw) {
            p.b = xs;
            p.ldb = up8(k);
            p.all = all;
            p.ld_all = ldx;
            p.rows = (int32_t)words;
            p.cols = (int32_t)k;
            p.depth = (int32_t)m;
            p.dynamic = 2;
            p.begins = p.ends = 1;
            p.scatter = 0;
            p.out = static_cast<uint16_t*>(dw) + c0 * k;
            p.ldo = k;
            const LossPlan q = planned(p, OP_DEPTH, OP_DEPTH, parts);
            if (launch_loss_sum(p, format, OP_DEPTH, q, stream) != hipSuccess) return EDKM_ERR_HIP;
        }
    }
    return EDKM_OK;
}

}  // extern "C"
