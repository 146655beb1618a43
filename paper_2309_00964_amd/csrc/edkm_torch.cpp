// Argument marshalling of the layer and optimizer calls for torch tensors, as a Python
// extension: checks, pointers and leading dimensions, and the differentiable product.
// It makes the same calls of libedkm.so as the ctypes binding (whose loaded library's
// addresses it is given) and does nothing else; a serving step's call costs a few
// microseconds of Python otherwise, as much as its kernel.

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/edkm.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <optional>
#include <stdexcept>
#include <vector>

namespace {

using at::Tensor;

struct Library {
    decltype(&edkm_linear_workspace_bytes) linear_ws;
    decltype(&edkm_linear) linear;
    decltype(&edkm_linear_backward_workspace_bytes) backward_ws;
    decltype(&edkm_linear_backward) backward;
    decltype(&edkm_palette_linear_workspace_bytes) palette_ws;
    decltype(&edkm_palette_linear) palette;
    decltype(&edkm_unpalettize) unpalettize;
    decltype(&edkm_adamw_batch) adamw;
    decltype(&edkm_embedding) embedding;
    decltype(&edkm_palette_embedding) palette_embedding;
    decltype(&edkm_embedding_backward_workspace_bytes) embedding_ws;
    decltype(&edkm_embedding_backward) embedding_backward;
    decltype(&edkm_residual_norm) norm;
    decltype(&edkm_residual_norm_backward_workspace_bytes) norm_ws;
    decltype(&edkm_residual_norm_backward) norm_backward;
    decltype(&edkm_linear_cross_entropy_workspace_bytes) loss_ws;
    decltype(&edkm_linear_cross_entropy) loss;
    decltype(&edkm_linear_cross_entropy_backward_workspace_bytes) loss_backward_ws;
    decltype(&edkm_linear_cross_entropy_backward) loss_backward;
    decltype(&edkm_status_str) status;
} lib;

// a refusal: ValueError in Python
[[noreturn]] __attribute__((format(printf, 1, 2))) void refuse(const char* fmt, ...) {
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    throw std::invalid_argument(text);
}

// a status of the library that is not EDKM_OK
struct Failed : std::exception {
    edkm_status status;
    const char* where;
    Failed(edkm_status s, const char* w) : status(s), where(w) {}
    const char* what() const noexcept override { return where; }
};
void check(edkm_status s, const char* where) {
    if (s != EDKM_OK) throw Failed(s, where);
}

const char* type_name(at::ScalarType t) { return c10::toString(t); }

int format_of(const Tensor& t, const char* name) {
    if (t.scalar_type() == at::kHalf) return EDKM_KEYS_FP16;
    if (t.scalar_type() == at::kBFloat16) return EDKM_KEYS_BF16;
    refuse("%s must be an fp16 or bf16 device tensor, not %s", name, type_name(t.scalar_type()));
}

void on_gpu(const Tensor& t, const char* name) {
    if (!t.is_cuda()) refuse("%s must be an fp16 or bf16 device tensor, not on %s", name, t.device().str().c_str());
}

void like(const Tensor& t, const Tensor& ref, const char* name) {
    if (t.scalar_type() != ref.scalar_type() || t.device() != ref.device())
        refuse("%s must have the type and device of the first tensor (%s, %s)", name, type_name(ref.scalar_type()),
               ref.device().str().c_str());
}

struct Matrix {
    void* p = nullptr;
    int64_t ld = 0;
};
// A rows x cols matrix of ref's type and device whose rows have no gaps and do not overlap.
Matrix matrix(const Tensor& t, int64_t rows, int64_t cols, const Tensor& ref, const char* name) {
    like(t, ref, name);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) {
        std::string s;
        for (auto d : t.sizes()) s += (s.empty() ? "" : "x") + std::to_string(d);
        refuse("%s must be %lld x %lld, not %s", name, (long long)rows, (long long)cols, s.c_str());
    }
    if ((t.stride(1) != 1 && cols > 1) || (t.stride(0) < cols && rows > 1))
        refuse("%s must have contiguous rows that do not overlap", name);
    return {t.data_ptr(), rows > 1 ? t.stride(0) : cols};
}
Matrix matrix(const Tensor* t, int64_t rows, int64_t cols, const Tensor& ref, const char* name) {
    return t ? matrix(*t, rows, cols, ref, name) : Matrix{nullptr, cols};
}
void* vec(const Tensor* t, int64_t count, const Tensor& ref, const char* name) {
    if (!t) return nullptr;
    like(*t, ref, name);
    if (t->numel() != count || !t->is_contiguous()) refuse("%s must hold %lld contiguous elements", name, (long long)count);
    return t->data_ptr();
}

// The stream of a call: the given one, or the tensors' device's current one.
hipStream_t stream_of(const Tensor& t, const hipStream_t* given) {
    return given ? *given : c10::hip::getCurrentHIPStream(t.get_device()).stream();
}

// The caller's workspace, or one from torch's allocator.  That one belongs to the current
// stream, so a call on another one has to bring its own.
struct Scratch {
    Tensor hold;
    void* p = nullptr;
    size_t bytes = 0;
    Scratch(const Tensor* ws, size_t need, const Tensor& ref, const hipStream_t* given) {
        if (ws) {
            if (ws->device() != ref.device() || !ws->is_contiguous())
                refuse("workspace must be a contiguous tensor on the operands' device");
            p = ws->data_ptr();
            bytes = ws->nbytes();
        } else if (need) {
            if (given && *given != c10::hip::getCurrentHIPStream(ref.get_device()).stream())
                refuse("a call on another stream than the current one needs a workspace of %zu bytes", need);
            hold = at::empty({(int64_t)need}, ref.options().dtype(at::kByte));
            p = hold.data_ptr();
            bytes = need;
        }
    }
};

void do_linear(const Tensor& x, const Tensor& w, const Tensor& y, const Tensor* bias, const Tensor* res, int act, const Tensor* z,
               const Tensor* ws, const hipStream_t* given) {
    const int fmt = format_of(x, "x");
    if (x.dim() != 2 || w.dim() != 2) refuse("x and w must be matrices");
    const int64_t m = x.size(0), k = x.size(1), n = w.size(0);
    const Matrix mx = matrix(x, m, k, x, "x"), mw = matrix(w, n, k, x, "w"), my = matrix(y, m, n, x, "y"),
                 mr = matrix(res, m, n, x, "residual");
    void *pb = vec(bias, n, x, "bias"), *pz = vec(z, m * n, x, "z_out");
    on_gpu(x, "x");
    c10::OptionalDeviceGuard guard(x.device());
    Scratch s(ws, lib.linear_ws(m, n, k), x, given);
    check(lib.linear(m, n, k, fmt, act, mx.p, mx.ld, mw.p, mw.ld, pb, mr.p, mr.ld, my.p, my.ld, pz, s.p, s.bytes, stream_of(x, given)),
          "linear");
}

void do_backward(const Tensor& dy, const Tensor* x, const Tensor* w, const Tensor* dx, const Tensor* dw, const Tensor* db, const Tensor* z,
                 int act, const Tensor* ws, const hipStream_t* given) {
    const int fmt = format_of(dy, "dy");
    if (dy.dim() != 2) refuse("dy must be a matrix");
    const int64_t m = dy.size(0), n = dy.size(1);
    if (!x && dw) refuse("dw needs x");
    if (!w && dx) refuse("dx needs w");
    if (act != EDKM_ACT_NONE && !z) refuse("an activation's backward needs z");
    int64_t k = 1;
    for (const Tensor* t : {x, w, dx, dw})
        if (t) {
            if (t->dim() != 2) refuse("x, w, dx and dw must be matrices");
            k = t->size(1);
            break;
        }
    const Matrix md = matrix(dy, m, n, dy, "dy"), mx = matrix(x, m, k, dy, "x"), mw = matrix(w, n, k, dy, "w"),
                 mdx = matrix(dx, m, k, dy, "dx");
    void *pdw = vec(dw, n * k, dy, "dw"), *pdb = vec(db, n, dy, "dbias"), *pz = vec(z, m * n, dy, "z");
    on_gpu(dy, "dy");
    c10::OptionalDeviceGuard guard(dy.device());
    Scratch s(ws, lib.backward_ws(m, n, k, act), dy, given);
    check(lib.backward(m, n, k, fmt, act, md.p, md.ld, pz, mx.p, mx.ld, mw.p, mw.ld, mdx.p, mdx.ld, pdw, pdb, s.p, s.bytes,
                       stream_of(dy, given)),
          "linear_backward");
}

// bits of a palette of `count` weights
int palette_bits(const Tensor& idx, const Tensor& lut, int64_t count, const Tensor& ref) {
    int bits = 0;
    while (bits < 5 && (1 << bits) < lut.numel()) ++bits;
    if (bits < 1 || bits > EDKM_MAX_BITS || lut.numel() != 1 << bits || lut.scalar_type() != at::kFloat || !lut.is_contiguous())
        refuse("lut must hold 2, 4, 8 or 16 contiguous float32 values");
    if (count > (int64_t)EDKM_MAX_N) refuse("a palette holds at most %llu weights", (unsigned long long)EDKM_MAX_N);
    const int64_t need = (count * bits + 7) / 8;
    if (idx.element_size() != 1 || !idx.is_contiguous() || idx.numel() < need) refuse("indices must be %lld contiguous bytes", (long long)need);
    if (idx.device() != ref.device() || lut.device() != ref.device())
        refuse("indices and lut must be on %s", ref.device().str().c_str());
    return bits;
}

void do_palette(const Tensor& x, const Tensor& idx, const Tensor& lut, const Tensor& y, const Tensor* bias, const Tensor* res, int act,
                const Tensor* z, const Tensor* ws, const hipStream_t* given) {
    const int fmt = format_of(x, "x");
    if (x.dim() != 2 || y.dim() != 2) refuse("x and y must be matrices");
    const int64_t m = x.size(0), k = x.size(1), n = y.size(1);
    const Matrix mx = matrix(x, m, k, x, "x"), my = matrix(y, m, n, x, "y"), mr = matrix(res, m, n, x, "residual");
    void *pb = vec(bias, n, x, "bias"), *pz = vec(z, m * n, x, "z_out");
    if (n > 0 && k > (int64_t)EDKM_MAX_N / n) refuse("a palette holds at most %llu weights", (unsigned long long)EDKM_MAX_N);
    const int bits = palette_bits(idx, lut, n * k, x);
    on_gpu(x, "x");
    c10::OptionalDeviceGuard guard(x.device());
    Scratch s(ws, lib.palette_ws(m, n, k, bits), x, given);
    check(lib.palette(m, n, k, bits, fmt, act, mx.p, mx.ld, (const uint8_t*)idx.data_ptr(), (const float*)lut.data_ptr(), pb, mr.p, mr.ld,
                      my.p, my.ld, pz, s.p, s.bytes, stream_of(x, given)),
          "palette_linear");
}

void do_unpalettize(const Tensor& idx, const Tensor& lut, const Tensor& w, const hipStream_t* given) {
    const int fmt = format_of(w, "w_out");
    if (!w.is_contiguous()) refuse("w_out must be contiguous");
    const int bits = palette_bits(idx, lut, w.numel(), w);
    on_gpu(w, "w_out");
    c10::OptionalDeviceGuard guard(w.device());
    check(lib.unpalettize((const uint8_t*)idx.data_ptr(), w.numel(), bits, fmt, (const float*)lut.data_ptr(), (uint16_t*)w.data_ptr(),
                          stream_of(w, given)),
          "unpalettize");
}

// Tokens or targets: int32 or int64, without gaps.
struct Index {
    const void* p;
    int type;
};
Index index_of(const Tensor& t, int64_t count, const Tensor& ref, const char* name) {
    if (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) refuse("%s must be int32 or int64, not %s", name, type_name(t.scalar_type()));
    if (t.device() != ref.device()) refuse("%s must be on %s", name, ref.device().str().c_str());
    if (t.numel() != count || !t.is_contiguous()) refuse("%s must hold %lld contiguous indices", name, (long long)count);
    return {t.data_ptr(), t.scalar_type() == at::kLong ? EDKM_INDEX_INT64 : EDKM_INDEX_INT32};
}
float* floats(const Tensor* t, int64_t count, const Tensor& ref, const char* name) {
    if (!t) return nullptr;
    if (t->scalar_type() != at::kFloat || t->device() != ref.device() || t->numel() != count || !t->is_contiguous())
        refuse("%s must hold %lld contiguous float32 values on %s", name, (long long)count, ref.device().str().c_str());
    return (float*)t->data_ptr();
}

void do_embedding(const Tensor& ids, const Tensor& table, const Tensor& y, double scale, const hipStream_t* given) {
    const int fmt = format_of(table, "table");
    if (table.dim() != 2) refuse("table must be a matrix");
    const int64_t m = ids.numel(), v = table.size(0), d = table.size(1);
    const Matrix mt = matrix(table, v, d, table, "table"), my = matrix(y, m, d, table, "y");
    const Index ix = index_of(ids, m, table, "ids");
    on_gpu(table, "table");
    c10::OptionalDeviceGuard guard(table.device());
    check(lib.embedding(m, v, d, fmt, ix.type, ix.p, mt.p, mt.ld, (float)scale, my.p, my.ld, stream_of(table, given)), "embedding");
}

void do_palette_embedding(const Tensor& ids, const Tensor& idx, const Tensor& lut, int64_t v, const Tensor& y, double scale,
                          const hipStream_t* given) {
    const int fmt = format_of(y, "y");
    if (y.dim() != 2) refuse("y must be a matrix");
    const int64_t m = ids.numel(), d = y.size(1);
    const Matrix my = matrix(y, m, d, y, "y");
    const Index ix = index_of(ids, m, y, "ids");
    if (v < 1 || d < 1) refuse("a palette's table has one row and one column at least");
    if (d > (int64_t)EDKM_MAX_N / v) refuse("a palette holds at most %llu weights", (unsigned long long)EDKM_MAX_N);
    const int bits = palette_bits(idx, lut, v * d, y);
    on_gpu(y, "y");
    c10::OptionalDeviceGuard guard(y.device());
    check(lib.palette_embedding(m, v, d, bits, fmt, ix.type, ix.p, (const uint8_t*)idx.data_ptr(), (const float*)lut.data_ptr(), (float)scale,
                                my.p, my.ld, stream_of(y, given)),
          "palette_embedding");
}

void do_embedding_backward(const Tensor& ids, const Tensor& dy, const Tensor& dt, double scale, bool accumulate, const Tensor* ws,
                           const hipStream_t* given) {
    const int fmt = format_of(dy, "dy");
    if (dt.dim() != 2) refuse("dtable must be a matrix");
    const int64_t m = ids.numel(), v = dt.size(0), d = dt.size(1);
    const Matrix mt = matrix(dt, v, d, dy, "dtable"), my = matrix(dy, m, d, dy, "dy");
    const Index ix = index_of(ids, m, dy, "ids");
    on_gpu(dy, "dy");
    c10::OptionalDeviceGuard guard(dy.device());
    Scratch s(ws, lib.embedding_ws(m, v, d), dy, given);
    check(lib.embedding_backward(m, v, d, fmt, ix.type, ix.p, my.p, my.ld, (float)scale, accumulate, mt.p, mt.ld, s.p, s.bytes,
                                 stream_of(dy, given)),
          "embedding_backward");
}

// A gate: n values, or a value for each of m x n.
struct Gate {
    Matrix m;
    int rows = 0;
};
Gate gate_of(const Tensor* gate, int64_t m, int64_t n, const Tensor& ref) {
    Gate g;
    if (!gate) return g;
    if (gate->dim() == 1) {
        g.m.p = vec(gate, n, ref, "gate");
    } else {
        g.m = matrix(*gate, m, n, ref, "gate");
        g.rows = 1;
    }
    return g;
}

void do_norm(const Tensor& r, const Tensor& w, const Tensor& y, const Tensor* h, const Tensor* u, const Tensor* post, const Tensor* gate,
             double scale, double eps, const hipStream_t* given) {
    const int fmt = format_of(r, "residual");
    if (r.dim() != 2) refuse("residual must be a matrix");
    const int64_t m = r.size(0), n = r.size(1);
    if (!u && (post || gate || h)) refuse("post_weight, gate and h belong to a block's output");
    if (u && !h) refuse("a block's output needs h");
    const Matrix mr = matrix(r, m, n, r, "residual"), my = matrix(y, m, n, r, "y"), mh = matrix(h, m, n, r, "h"), mu = matrix(u, m, n, r, "block");
    const void *pw = vec(&w, n, r, "weight"), *pp = vec(post, n, r, "post_weight");
    const Gate g = gate_of(gate, m, n, r);
    on_gpu(r, "residual");
    c10::OptionalDeviceGuard guard(r.device());
    check(lib.norm(m, n, fmt, mr.p, mr.ld, mu.p, mu.ld, pw, pp, g.m.p, g.m.ld, g.rows, (float)scale, (float)eps, mh.p, mh.ld, my.p, my.ld,
                   stream_of(r, given)),
          "residual_norm");
}

void do_norm_backward(const Tensor* dy, const Tensor* dh, const Tensor& r, const Tensor* u, const Tensor& w, const Tensor* post,
                      const Tensor* gate, double scale, double eps, const Tensor* dr, const Tensor* du, const Tensor* dw, const Tensor* dpost,
                      const Tensor* dgate, const Tensor* ws, const hipStream_t* given) {
    const int fmt = format_of(r, "residual");
    if (r.dim() != 2) refuse("residual must be a matrix");
    const int64_t m = r.size(0), n = r.size(1);
    if (!u && (post || gate || du)) refuse("post_weight, gate and dblock belong to a block's output");
    if ((dpost && !post) || (dgate && !gate)) refuse("a gradient of what is not given");
    const Matrix mr = matrix(r, m, n, r, "residual"), mdy = matrix(dy, m, n, r, "dy"), mdh = matrix(dh, m, n, r, "dh"), mu = matrix(u, m, n, r, "block"),
                 mdr = matrix(dr, m, n, r, "dresidual"), mdu = matrix(du, m, n, r, "dblock");
    const void *pw = vec(&w, n, r, "weight"), *pp = vec(post, n, r, "post_weight");
    const Gate g = gate_of(gate, m, n, r);
    void *pdw = vec(dw, n, r, "dweight"), *pdp = vec(dpost, n, r, "dpost_weight"), *pdg = vec(dgate, g.rows ? m * n : n, r, "dgate");
    on_gpu(r, "residual");
    c10::OptionalDeviceGuard guard(r.device());
    Scratch s(ws, lib.norm_ws(m, n), r, given);
    check(lib.norm_backward(m, n, fmt, mdy.p, mdy.ld, mdh.p, mdh.ld, mr.p, mr.ld, mu.p, mu.ld, pw, pp, g.m.p, g.m.ld, g.rows, (float)scale,
                            (float)eps, mdr.p, mdr.ld, mdu.p, mdu.ld, pdw, pdp, pdg, s.p, s.bytes, stream_of(r, given)),
          "residual_norm_backward");
}

void do_loss(const Tensor& x, const Tensor& w, const Tensor& targets, const Tensor& loss, const Tensor* lse, int reduction, const Tensor* ws,
             const hipStream_t* given) {
    const int fmt = format_of(x, "x");
    if (x.dim() != 2 || w.dim() != 2) refuse("x and w must be matrices");
    const int64_t m = x.size(0), k = x.size(1), n = w.size(0);
    const Matrix mx = matrix(x, m, k, x, "x"), mw = matrix(w, n, k, x, "w");
    const Index ix = index_of(targets, m, x, "targets");
    float *pl = floats(&loss, reduction == EDKM_REDUCE_NONE ? m : 1, x, "loss"), *pe = floats(lse, m, x, "lse");
    on_gpu(x, "x");
    c10::OptionalDeviceGuard guard(x.device());
    Scratch s(ws, lib.loss_ws(m, n, k), x, given);
    check(lib.loss(m, n, k, fmt, ix.type, reduction, mx.p, mx.ld, mw.p, mw.ld, ix.p, pl, pe, s.p, s.bytes, stream_of(x, given)),
          "linear_cross_entropy");
}

void do_loss_backward(const Tensor& dloss, const Tensor& x, const Tensor& w, const Tensor& targets, const Tensor& lse, const Tensor* dx,
                      const Tensor* dw, int reduction, const Tensor* ws, const hipStream_t* given) {
    const int fmt = format_of(x, "x");
    if (x.dim() != 2 || w.dim() != 2) refuse("x and w must be matrices");
    const int64_t m = x.size(0), k = x.size(1), n = w.size(0);
    const Matrix mx = matrix(x, m, k, x, "x"), mw = matrix(w, n, k, x, "w"), mdx = matrix(dx, m, k, x, "dx");
    const Index ix = index_of(targets, m, x, "targets");
    float *pg = floats(&dloss, reduction == EDKM_REDUCE_NONE ? m : 1, x, "dloss"), *pe = floats(&lse, m, x, "lse");
    void* pdw = vec(dw, n * k, x, "dw");
    on_gpu(x, "x");
    c10::OptionalDeviceGuard guard(x.device());
    Scratch s(ws, lib.loss_backward_ws(m, n, k), x, given);
    check(lib.loss_backward(m, n, k, fmt, ix.type, reduction, pg, mx.p, mx.ld, mw.p, mw.ld, ix.p, pe, mdx.p, mdx.ld, pdw, s.p, s.bytes,
                            stream_of(x, given)),
          "linear_cross_entropy_backward");
}

// ---------------------------------------------------------------------------
// differentiable forms

// A tensor of any leading shape as a matrix whose rows have no gaps.
Tensor rows_of(const Tensor& t, int64_t cols) {
    Tensor m = t.dim() == 2 ? t : t.reshape({-1, cols});
    const bool ok = (m.stride(1) == 1 || cols == 1) && (m.stride(0) >= cols || m.size(0) <= 1);
    return ok ? m : m.contiguous();
}

struct Shapes {
    std::vector<int64_t> out;
    int64_t k;
};
Shapes shapes_of(const Tensor& x, int64_t n, const Tensor* bias, const Tensor* res) {
    format_of(x, "x");
    on_gpu(x, "x");
    Shapes s;
    s.k = x.size(-1);
    s.out.assign(x.sizes().begin(), x.sizes().end());
    s.out.back() = n;
    if (bias) like(*bias, x, "bias");
    if (res) like(*res, x, "residual");
    return s;
}

struct Operands {
    Tensor x2, r2, b, y, z;
    Operands(const Tensor& x, const Tensor* bias, const Tensor* res, int64_t n, const Shapes& s, bool keep_z) {
        x2 = rows_of(x, s.k);
        if (res) r2 = rows_of(*res, n);
        if (bias) b = bias->contiguous();
        y = at::empty(s.out, x.options());
        if (keep_z) z = at::empty({x2.size(0), n}, x.options());
    }
    const Tensor* bias() const { return b.defined() ? &b : nullptr; }
    const Tensor* res() const { return r2.defined() ? &r2 : nullptr; }
    const Tensor* keep() const { return z.defined() ? &z : nullptr; }
    Tensor rows(int64_t n) const { return y.dim() == 2 ? y : y.view({-1, n}); }
};

using torch::autograd::AutogradContext;
using torch::autograd::Variable;
using torch::autograd::variable_list;

// A gradient that cannot be differentiated again says so when that is tried.
void once(variable_list& g, const char* why = "the product's gradients cannot be differentiated again") {
    if (!at::GradMode::is_enabled()) return;
    variable_list there;
    for (auto& t : g)
        if (t.defined()) there.push_back(t.detach().requires_grad_(true));
    auto node = std::make_shared<torch::autograd::DelayedError>(why, (int)there.size());
    node->set_next_edges(torch::autograd::collect_next_edges(there));
    there = node->apply(std::move(there));
    size_t i = 0;
    for (auto& t : g)
        if (t.defined()) t = there[i++];
}

typedef std::optional<Tensor> Maybe;
const Tensor* get(const Maybe& t) { return t ? &*t : nullptr; }

struct LinearFunction : torch::autograd::Function<LinearFunction> {
    static Variable forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, const Maybe& bias, const Maybe& res, int64_t act, bool grad) {
        const int64_t n = w.size(0);
        const bool gx = grad && x.requires_grad(), gw = grad && w.requires_grad(), gb = grad && bias && bias->requires_grad(),
                   gr = grad && res && res->requires_grad();
        at::AutoDispatchBelowADInplaceOrView below;
        const Shapes s = shapes_of(x, n, get(bias), get(res));
        Operands o(x, get(bias), get(res), n, s, act != EDKM_ACT_NONE && (gx || gw || gb));
        const Tensor w2 = rows_of(w, s.k);
        do_linear(o.x2, w2, o.rows(n), o.bias(), o.res(), (int)act, o.keep(), nullptr, nullptr);
        // x and w themselves are saved too, for autograd's check that they are unchanged
        ctx->save_for_backward({gw ? x : Tensor(), gx ? w : Tensor(), o.z});
        ctx->saved_data["n"] = n;
        ctx->saved_data["act"] = act;
        ctx->saved_data["need"] = (int64_t)(gx | gw << 1 | gb << 2 | gr << 3);
        ctx->saved_data["shape"] = x.sizes().vec();
        return o.y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const int64_t n = ctx->saved_data["n"].toInt(), need = ctx->saved_data["need"].toInt();
        const auto shape = ctx->saved_data["shape"].toIntVector();
        const int act = (int)ctx->saved_data["act"].toInt();
        variable_list out(6);
        if (!grads[0].defined()) return out;
        const int64_t k = shape.back();
        {
            at::AutoDispatchBelowADInplaceOrView below;
            const Tensor dy = rows_of(grads[0], n);
            Tensor x2, w2, dw;
            if ((need & 1) && ctx->needs_input_grad(0)) {
                out[0] = at::empty(shape, dy.options());
                w2 = rows_of(saved[1], k);
            }
            if ((need & 2) && ctx->needs_input_grad(1)) {
                out[1] = at::empty({n, k}, dy.options());
                x2 = rows_of(saved[0], k);
            }
            if (need & 4) out[2] = at::empty({n}, dy.options());
            if (out[0].defined() || out[1].defined() || out[2].defined()) {
                Tensor dx = out[0].defined() ? (out[0].dim() == 2 ? out[0] : out[0].view({-1, k})) : Tensor();
                do_backward(dy, x2.defined() ? &x2 : nullptr, w2.defined() ? &w2 : nullptr, dx.defined() ? &dx : nullptr,
                            out[1].defined() ? &out[1] : nullptr, out[2].defined() ? &out[2] : nullptr,
                            saved[2].defined() ? &saved[2] : nullptr, act, nullptr, nullptr);
            }
        }
        once(out);
        if (need & 8) out[3] = grads[0];
        return out;
    }
};

struct PaletteFunction : torch::autograd::Function<PaletteFunction> {
    static Variable forward(AutogradContext* ctx, const Tensor& x, const Maybe& bias, const Maybe& res, const Tensor& idx,
                            const Tensor& lut, int64_t n, int64_t act) {
        const bool gx = x.requires_grad(), gb = bias && bias->requires_grad(), gr = res && res->requires_grad();
        at::AutoDispatchBelowADInplaceOrView below;
        const Shapes s = shapes_of(x, n, get(bias), get(res));
        Operands o(x, get(bias), get(res), n, s, act != EDKM_ACT_NONE && (gx || gb));
        do_palette(o.x2, idx, lut, o.rows(n), o.bias(), o.res(), (int)act, o.keep(), nullptr, nullptr);
        ctx->save_for_backward({idx, lut, o.z});
        ctx->saved_data["n"] = n;
        ctx->saved_data["act"] = act;
        ctx->saved_data["need"] = (int64_t)(gx | gb << 1 | gr << 2);
        ctx->saved_data["shape"] = x.sizes().vec();
        return o.y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const auto saved = ctx->get_saved_variables();
        const int64_t n = ctx->saved_data["n"].toInt(), need = ctx->saved_data["need"].toInt();
        const auto shape = ctx->saved_data["shape"].toIntVector();
        const int act = (int)ctx->saved_data["act"].toInt();
        variable_list out(7);
        if (!grads[0].defined()) return out;
        const int64_t k = shape.back();
        {
            at::AutoDispatchBelowADInplaceOrView below;
            const Tensor dy = rows_of(grads[0], n);
            Tensor w, dx;
            if (need & 1) {
                w = at::empty({n, k}, dy.options());
                do_unpalettize(saved[0], saved[1], w, nullptr);
                out[0] = at::empty(shape, dy.options());
                dx = out[0].dim() == 2 ? out[0] : out[0].view({-1, k});
            }
            if (need & 2) out[1] = at::empty({n}, dy.options());
            if (need & 3)
                do_backward(dy, nullptr, w.defined() ? &w : nullptr, dx.defined() ? &dx : nullptr, nullptr,
                            out[1].defined() ? &out[1] : nullptr, saved[2].defined() ? &saved[2] : nullptr, act, nullptr, nullptr);
        }
        once(out);
        if (need & 4) out[2] = grads[0];
        return out;
    }
};

Tensor as_rows(const Tensor& t, int64_t n) { return t.dim() == 2 ? t : t.view({-1, n}); }

struct EmbeddingFunction : torch::autograd::Function<EmbeddingFunction> {
    static Variable forward(AutogradContext* ctx, const Tensor& table, const Tensor& ids, double scale) {
        at::AutoDispatchBelowADInplaceOrView below;
        const int64_t d = table.size(1);
        auto shape = ids.sizes().vec();
        shape.push_back(d);
        Tensor y = at::empty(shape, table.options());
        do_embedding(ids.contiguous(), rows_of(table, d), y.dim() == 2 ? y : y.view({ids.numel(), d}), scale, nullptr);
        ctx->save_for_backward({ids});
        ctx->saved_data["v"] = table.size(0);
        ctx->saved_data["d"] = d;
        ctx->saved_data["scale"] = scale;
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        variable_list out(3);
        if (!grads[0].defined()) return out;
        const auto saved = ctx->get_saved_variables();
        const int64_t v = ctx->saved_data["v"].toInt(), d = ctx->saved_data["d"].toInt();
        {
            at::AutoDispatchBelowADInplaceOrView below;
            const Tensor ids = saved[0].contiguous();
            Tensor dy = grads[0];
            dy = dy.dim() == 2 ? rows_of(dy, d) : rows_of(dy.reshape({ids.numel(), d}), d);
            out[0] = at::empty({v, d}, dy.options());
            do_embedding_backward(ids, dy, out[0], ctx->saved_data["scale"].toDouble(), false, nullptr, nullptr);
        }
        once(out, "the embedding's gradient cannot be differentiated again");
        return out;
    }
};

struct LossFunction : torch::autograd::Function<LossFunction> {
    static Variable forward(AutogradContext* ctx, const Tensor& x, const Tensor& w, const Tensor& targets, int64_t reduction) {
        at::AutoDispatchBelowADInplaceOrView below;
        const int64_t k = x.size(-1);
        const Tensor x2 = rows_of(x, k), w2 = rows_of(w, k);
        const auto o = x.options().dtype(at::kFloat);
        Tensor loss = reduction == EDKM_REDUCE_NONE ? at::empty(targets.sizes(), o) : at::empty({}, o), lse = at::empty({x2.size(0)}, o);
        do_loss(x2, w2, targets.contiguous(), loss, &lse, (int)reduction, nullptr, nullptr);
        ctx->save_for_backward({x, w, targets, lse});
        ctx->saved_data["reduction"] = reduction;
        return loss;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        variable_list out(4);
        if (!grads[0].defined()) return out;
        const auto saved = ctx->get_saved_variables();
        const Tensor &x = saved[0], &w = saved[1];
        const int64_t k = x.size(-1);
        {
            at::AutoDispatchBelowADInplaceOrView below;
            Tensor dx;
            if (ctx->needs_input_grad(0)) {
                out[0] = at::empty(x.sizes(), x.options());
                dx = as_rows(out[0], k);
            }
            if (ctx->needs_input_grad(1)) out[1] = at::empty(w.sizes(), w.options());
            if (dx.defined() || out[1].defined())
                do_loss_backward(grads[0].contiguous(), rows_of(x, k), rows_of(w, k), saved[2].contiguous(), saved[3], dx.defined() ? &dx : nullptr,
                                 out[1].defined() ? &out[1] : nullptr, (int)ctx->saved_data["reduction"].toInt(), nullptr, nullptr);
        }
        once(out, "the cross entropy's gradients cannot be differentiated again");
        return out;
    }
};

// h and y, or y alone without a block's output.
struct NormFunction : torch::autograd::Function<NormFunction> {
    static variable_list forward(AutogradContext* ctx, const Tensor& r, const Tensor& w, const Maybe& u, const Maybe& post, const Maybe& gate,
                                 double scale, double eps) {
        at::AutoDispatchBelowADInplaceOrView below;
        const int64_t n = r.size(-1);
        const Tensor r2 = rows_of(r, n), w1 = w.contiguous();
        Tensor y = at::empty(r.sizes(), r.options()), h, h2, u2, p1, g2;
        if (u) {
            h = at::empty(r.sizes(), r.options());
            h2 = as_rows(h, n);
            u2 = rows_of(*u, n);
        }
        if (post) p1 = post->contiguous();
        if (gate) g2 = gate->dim() == 1 && r.dim() > 1 ? gate->contiguous() : gate_rows(*gate, n);
        do_norm(r2, w1, as_rows(y, n), h.defined() ? &h2 : nullptr, u ? &u2 : nullptr, post ? &p1 : nullptr, gate ? &g2 : nullptr, scale, eps,
                nullptr);
        ctx->save_for_backward({r, w, u ? *u : Tensor(), post ? *post : Tensor(), gate ? *gate : Tensor()});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["eps"] = eps;
        ctx->set_materialize_grads(false);
        return u ? variable_list{h, y} : variable_list{y};
    }
    // a single row's gate may be a vector; more rows' is one for each
    static Tensor gate_rows(const Tensor& gate, int64_t n) { return gate.dim() == 1 ? gate.contiguous() : rows_of(gate, n); }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        variable_list out(7);
        const auto saved = ctx->get_saved_variables();
        const Tensor &r = saved[0], &w = saved[1], &u = saved[2], &post = saved[3], &gate = saved[4];
        const Tensor& gy = grads.back();
        const Tensor gh = u.defined() ? grads[0] : Tensor();
        if (!gy.defined() && !gh.defined()) return out;
        const int64_t n = r.size(-1);
        {
            at::AutoDispatchBelowADInplaceOrView below;
            Tensor dy, dh, u2, p1, g2, dr, du;
            if (gy.defined()) dy = rows_of(gy, n);
            if (gh.defined()) dh = rows_of(gh, n);
            if (u.defined()) u2 = rows_of(u, n);
            if (post.defined()) p1 = post.contiguous();
            if (gate.defined()) g2 = gate_rows(gate, n);
            const Tensor* in[] = {&r, &w, &u, &post, &gate};
            bool any = false;
            for (int i = 0, edge = 0; i < 5; ++i)      // autograd numbers the tensors that were given
                if (in[i]->defined() && ctx->needs_input_grad(edge++)) {
                    out[i] = at::empty(in[i]->sizes(), in[i]->options().memory_format(at::MemoryFormat::Contiguous));
                    any = true;
                }
            if (!any) return out;
            if (out[0].defined()) dr = as_rows(out[0], n);
            if (out[2].defined()) du = as_rows(out[2], n);
            auto at_ = [](const Tensor& t) { return t.defined() ? &t : nullptr; };
            do_norm_backward(at_(dy), at_(dh), rows_of(r, n), at_(u2), w.contiguous(), at_(p1), at_(g2), ctx->saved_data["scale"].toDouble(),
                             ctx->saved_data["eps"].toDouble(), at_(dr), at_(du), at_(out[1]), at_(out[3]), at_(out[4]), nullptr, nullptr);
        }
        once(out, "the norm's gradients cannot be differentiated again");
        return out;
    }
};

// ---------------------------------------------------------------------------
// optimizer

struct List {
    std::vector<void*> p;
    at::ScalarType type = at::kFloat;
};
// Pointers of contiguous tensors of one type that hold at least sizes[i] elements.
List pointers(PyObject* seq, const char* name, const std::vector<uint64_t>& sizes, std::initializer_list<at::ScalarType> types,
              at::Device device) {
    List out;
    PyObject* fast = PySequence_Fast(seq, "a list of tensors is wanted");
    if (!fast) throw python_error();
    struct Drop {
        PyObject* o;
        ~Drop() { Py_DECREF(o); }
    } drop{fast};
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(fast);
    if ((size_t)count != sizes.size()) refuse("%s has %zd entries for %zu parameters", name, count, sizes.size());
    out.p.resize(count);
    for (Py_ssize_t i = 0; i < count; ++i) {
        PyObject* o = PySequence_Fast_GET_ITEM(fast, i);
        if (!THPVariable_Check(o)) refuse("%s[%zd] is no tensor", name, i);
        const Tensor& t = THPVariable_Unpack(o);
        if (i == 0) out.type = t.scalar_type();
        bool known = t.scalar_type() == out.type;
        if (known && i == 0) known = std::find(types.begin(), types.end(), out.type) != types.end();
        if (!known) refuse("%s[%zd]: the type %s does not fit", name, i, type_name(t.scalar_type()));
        if (t.device() != device || !t.is_contiguous()) refuse("%s[%zd] must be contiguous and on the parameters' device", name, i);
        if ((uint64_t)t.numel() < sizes[i])
            refuse("%s[%zd] has %lld elements, %llu needed", name, i, (long long)t.numel(), (unsigned long long)sizes[i]);
        out.p[i] = t.data_ptr();
    }
    return out;
}

int param_type(at::ScalarType t) { return t == at::kHalf ? EDKM_TYPE_FP16 : t == at::kBFloat16 ? EDKM_TYPE_BF16 : EDKM_TYPE_FP32; }

// ---------------------------------------------------------------------------
// Python

const Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse("%s must be a tensor", name);
    return THPVariable_Unpack(o);
}
const Tensor* maybe(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
struct Given {
    hipStream_t s = nullptr;
    bool there = false;
    explicit Given(PyObject* o) {
        if (o == Py_None) return;
        there = true;
        s = (hipStream_t)(uintptr_t)PyLong_AsUnsignedLongLong(o);
        if (PyErr_Occurred()) throw python_error();
    }
    const hipStream_t* get() const { return there ? &s : nullptr; }
};

PyObject* error_type = nullptr;   // edkm.EdkmError(status, where)

template <class Fn>
PyObject* guarded(Py_ssize_t have, Py_ssize_t want, Fn fn) {
    if (have != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments wanted, %zd given", want, have);
        return nullptr;
    }
    try {
        return fn();
    } catch (const std::invalid_argument& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Failed& e) {
        PyObject* v = error_type ? PyObject_CallFunction(error_type, "is", (int)e.status, e.where) : nullptr;
        if (v) {
            PyErr_SetObject(error_type, v);
            Py_DECREF(v);
        } else if (!PyErr_Occurred()) {
            PyErr_SetString(PyExc_RuntimeError, e.where);
        }
    } catch (python_error& e) {
        e.persist();
        e.restore();
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::bad_alloc&) {
        PyErr_NoMemory();
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 2, [&]() -> PyObject* {
        auto at = [&](const char* name) {
            PyObject* v = PyDict_GetItemString(a[0], name);
            if (!v) refuse("no address of %s", name);
            return (void*)(uintptr_t)PyLong_AsUnsignedLongLong(v);
        };
        lib.linear_ws = (decltype(lib.linear_ws))at("edkm_linear_workspace_bytes");
        lib.linear = (decltype(lib.linear))at("edkm_linear");
        lib.backward_ws = (decltype(lib.backward_ws))at("edkm_linear_backward_workspace_bytes");
        lib.backward = (decltype(lib.backward))at("edkm_linear_backward");
        lib.palette_ws = (decltype(lib.palette_ws))at("edkm_palette_linear_workspace_bytes");
        lib.palette = (decltype(lib.palette))at("edkm_palette_linear");
        lib.unpalettize = (decltype(lib.unpalettize))at("edkm_unpalettize");
        lib.adamw = (decltype(lib.adamw))at("edkm_adamw_batch");
        lib.embedding = (decltype(lib.embedding))at("edkm_embedding");
        lib.palette_embedding = (decltype(lib.palette_embedding))at("edkm_palette_embedding");
        lib.embedding_ws = (decltype(lib.embedding_ws))at("edkm_embedding_backward_workspace_bytes");
        lib.embedding_backward = (decltype(lib.embedding_backward))at("edkm_embedding_backward");
        lib.norm = (decltype(lib.norm))at("edkm_residual_norm");
        lib.norm_ws = (decltype(lib.norm_ws))at("edkm_residual_norm_backward_workspace_bytes");
        lib.norm_backward = (decltype(lib.norm_backward))at("edkm_residual_norm_backward");
        lib.loss_ws = (decltype(lib.loss_ws))at("edkm_linear_cross_entropy_workspace_bytes");
        lib.loss = (decltype(lib.loss))at("edkm_linear_cross_entropy");
        lib.loss_backward_ws = (decltype(lib.loss_backward_ws))at("edkm_linear_cross_entropy_backward_workspace_bytes");
        lib.loss_backward = (decltype(lib.loss_backward))at("edkm_linear_cross_entropy_backward");
        lib.status = (decltype(lib.status))at("edkm_status_str");
        Py_INCREF(a[1]);
        Py_XSETREF(error_type, a[1]);
        Py_RETURN_NONE;
    });
}

// linear(x, w, y, bias, residual, activation, z, workspace, stream)
PyObject* py_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> PyObject* {
        do_linear(tensor(a[0], "x"), tensor(a[1], "w"), tensor(a[2], "y"), maybe(a[3], "bias"), maybe(a[4], "residual"), (int)integer(a[5]),
                  maybe(a[6], "z_out"), maybe(a[7], "workspace"), Given(a[8]).get());
        Py_RETURN_NONE;
    });
}

// linear_backward(dy, x, w, dx, dw, dbias, z, activation, workspace, stream)
PyObject* py_linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> PyObject* {
        do_backward(tensor(a[0], "dy"), maybe(a[1], "x"), maybe(a[2], "w"), maybe(a[3], "dx"), maybe(a[4], "dw"), maybe(a[5], "dbias"),
                    maybe(a[6], "z"), (int)integer(a[7]), maybe(a[8], "workspace"), Given(a[9]).get());
        Py_RETURN_NONE;
    });
}

// palette_linear(x, indices, lut, y, bias, residual, activation, z, workspace, stream)
PyObject* py_palette_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> PyObject* {
        do_palette(tensor(a[0], "x"), tensor(a[1], "indices"), tensor(a[2], "lut"), tensor(a[3], "y"), maybe(a[4], "bias"),
                   maybe(a[5], "residual"), (int)integer(a[6]), maybe(a[7], "z_out"), maybe(a[8], "workspace"), Given(a[9]).get());
        Py_RETURN_NONE;
    });
}

// unpalettize(indices, lut, w_out, stream)
PyObject* py_unpalettize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject* {
        do_unpalettize(tensor(a[0], "indices"), tensor(a[1], "lut"), tensor(a[2], "w_out"), Given(a[3]).get());
        Py_RETURN_NONE;
    });
}

void fits(const Tensor& x, int64_t n, const Tensor* bias, const Tensor* res) {
    if (x.dim() < 1) refuse("x needs a last dimension of inputs");
    if (bias && (bias->dim() != 1 || bias->size(0) != n)) refuse("bias must hold %lld elements", (long long)n);
    if (res) {
        bool ok = res->dim() == x.dim() && res->size(-1) == n;
        for (int64_t i = 0; ok && i + 1 < x.dim(); ++i) ok = res->size(i) == x.size(i);
        if (!ok) refuse("residual must have the output's shape");
    }
}

// apply_linear(x, w, bias, residual, activation) -> y
PyObject* py_apply_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject* {
        const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w");
        const Tensor *bias = maybe(a[2], "bias"), *res = maybe(a[3], "residual");
        if (x.dim() < 1 || w.dim() != 2 || x.size(-1) != w.size(1)) refuse("w must be n x k for x of (..., k)");
        fits(x, w.size(0), bias, res);
        Tensor y = LinearFunction::apply(x, w, bias ? Maybe(*bias) : Maybe(), res ? Maybe(*res) : Maybe(), integer(a[4]), at::GradMode::is_enabled());
        return THPVariable_Wrap(y);
    });
}

// apply_palette_linear(x, indices, lut, n, bias, residual, activation) -> y
PyObject* py_apply_palette_linear(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded(n_args, 7, [&]() -> PyObject* {
        const Tensor &x = tensor(a[0], "x"), &idx = tensor(a[1], "indices"), &lut = tensor(a[2], "lut");
        const int64_t n = integer(a[3]), act = integer(a[6]);
        const Tensor *bias = maybe(a[4], "bias"), *res = maybe(a[5], "residual");
        if (lut.requires_grad() && at::GradMode::is_enabled())
            refuse("a palette's table takes no gradient; train the weights through dkm and linear");
        if (n < 1) refuse("out_features must be 1 at least");
        fits(x, n, bias, res);
        // without reverse mode autograd is passed by, so its own refusal of tangents does not come
        for (const Tensor* t : {&x, &lut, bias, res})
            TORCH_CHECK(!t || !t->_fw_grad(0).defined(), "palette_linear: forward-mode derivatives are not implemented");
        const bool grad = at::GradMode::is_enabled() &&
                          (x.requires_grad() || (bias && bias->requires_grad()) || (res && res->requires_grad()));
        Tensor y;
        if (grad) {
            y = PaletteFunction::apply(x, bias ? Maybe(*bias) : Maybe(), res ? Maybe(*res) : Maybe(), idx, lut, n, act);
        } else {
            at::AutoDispatchBelowADInplaceOrView below;
            const Shapes s = shapes_of(x, n, bias, res);
            Operands o(x, bias, res, n, s, false);
            do_palette(o.x2, idx, lut, o.rows(n), o.bias(), o.res(), (int)act, nullptr, nullptr, nullptr);
            y = o.y;
        }
        return THPVariable_Wrap(y);
    });
}

// adamw_batch(params, grads, exp_avgs, exp_avg_sqs, step, lr, beta1, beta2, eps, weight_decay, masters, m_scales,
//             v_scales, seed, stream)
PyObject* py_adamw_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 15, [&]() -> PyObject* {
        PyObject* fast = PySequence_Fast(a[0], "params must be a list of tensors");
        if (!fast) throw python_error();
        std::vector<uint64_t> sizes(PySequence_Fast_GET_SIZE(fast));
        at::Device device(at::kCPU);
        Tensor first;
        for (size_t i = 0; i < sizes.size(); ++i) {
            PyObject* o = PySequence_Fast_GET_ITEM(fast, i);
            if (!THPVariable_Check(o)) {
                Py_DECREF(fast);
                refuse("params[%zu] is no tensor", i);
            }
            const Tensor& t = THPVariable_Unpack(o);
            sizes[i] = t.numel();
            if (i == 0) {
                device = t.device();
                first = t;
            }
        }
        Py_DECREF(fast);
        if (sizes.empty()) Py_RETURN_NONE;
        const List p = pointers(a[0], "params", sizes, {at::kHalf, at::kBFloat16, at::kFloat}, device);
        const List g = pointers(a[1], "grads", sizes, {p.type, at::kFloat}, device);
        if ((a[11] == Py_None) != (a[12] == Py_None)) refuse("8-bit states need m_scales and v_scales");
        const bool s8 = a[11] != Py_None;
        const List m = pointers(a[2], "exp_avgs", sizes, {s8 ? at::kFloat8_e4m3fn : at::kFloat}, device);
        const List v = pointers(a[3], "exp_avg_sqs", sizes, {s8 ? at::kFloat8_e5m2 : at::kFloat}, device);
        List w, ms, vs;
        if (s8) {
            std::vector<uint64_t> blocks(sizes.size());
            for (size_t i = 0; i < sizes.size(); ++i) blocks[i] = (sizes[i] + EDKM_STATE_BLOCK - 1) / EDKM_STATE_BLOCK;
            ms = pointers(a[11], "m_scales", blocks, {at::kFloat}, device);
            vs = pointers(a[12], "v_scales", blocks, {at::kFloat}, device);
        }
        if (a[10] != Py_None) {
            if (p.type == at::kFloat) refuse("float32 parameters take no masters");
            w = pointers(a[10], "masters", sizes, {at::kFloat}, device);
        }
        std::vector<std::pair<uintptr_t, uintptr_t>> spans;
        for (size_t i = 0; i < sizes.size(); ++i)
            if (sizes[i]) spans.emplace_back((uintptr_t)p.p[i], (uintptr_t)p.p[i] + sizes[i] * c10::elementSize(p.type));
        std::sort(spans.begin(), spans.end());
        for (size_t i = 1; i < spans.size(); ++i)
            if (spans[i].first < spans[i - 1].second) refuse("params: the same tensor twice, or two that overlap");
        const Tensor& step = tensor(a[4], "step");
        if (step.scalar_type() != at::kInt || step.numel() != 1 || step.device() != device)
            refuse("step must be one int32 on the parameters' device");
        const float* lr_dev = nullptr;
        double lr = 0;
        if (THPVariable_Check(a[5])) {
            const Tensor& t = THPVariable_Unpack(a[5]);
            if (t.scalar_type() != at::kFloat || t.numel() != 1 || t.device() != device)
                refuse("a tensor lr must be one float32 on the parameters' device");
            lr_dev = (const float*)t.data_ptr();
        } else {
            lr = number(a[5]);
        }
        const Given given(a[14]);
        if (device.type() != at::kCUDA) refuse("params must be device tensors, not on %s", device.str().c_str());
        c10::OptionalDeviceGuard guard(device);
        check(lib.adamw((int)sizes.size(), sizes.data(), param_type(p.type), param_type(g.type), s8 ? 8 : 32, p.p.data(),
                        w.p.empty() ? nullptr : (float* const*)w.p.data(), g.p.data(), m.p.data(), v.p.data(),
                        s8 ? (float* const*)ms.p.data() : nullptr, s8 ? (float* const*)vs.p.data() : nullptr, (int32_t*)step.data_ptr(),
                        lr_dev, lr, number(a[6]), number(a[7]), number(a[8]), number(a[9]), (uint32_t)(integer(a[13]) & 0xFFFFFFFF),
                        stream_of(first, given.get())),
              "adamw_batch");
        Py_RETURN_NONE;
    });
}

// embedding(ids, table, y, scale, stream)
PyObject* py_embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject* {
        do_embedding(tensor(a[0], "ids"), tensor(a[1], "table"), tensor(a[2], "y"), number(a[3]), Given(a[4]).get());
        Py_RETURN_NONE;
    });
}

// palette_embedding(ids, indices, lut, rows, y, scale, stream)
PyObject* py_palette_embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject* {
        do_palette_embedding(tensor(a[0], "ids"), tensor(a[1], "indices"), tensor(a[2], "lut"), integer(a[3]), tensor(a[4], "y"), number(a[5]),
                             Given(a[6]).get());
        Py_RETURN_NONE;
    });
}

// embedding_backward(ids, dy, dtable, scale, accumulate, workspace, stream)
PyObject* py_embedding_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject* {
        do_embedding_backward(tensor(a[0], "ids"), tensor(a[1], "dy"), tensor(a[2], "dtable"), number(a[3]), integer(a[4]) != 0,
                              maybe(a[5], "workspace"), Given(a[6]).get());
        Py_RETURN_NONE;
    });
}

// residual_norm(residual, weight, y, h, block, post_weight, gate, scale, eps, stream)
PyObject* py_residual_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> PyObject* {
        do_norm(tensor(a[0], "residual"), tensor(a[1], "weight"), tensor(a[2], "y"), maybe(a[3], "h"), maybe(a[4], "block"),
                maybe(a[5], "post_weight"), maybe(a[6], "gate"), number(a[7]), number(a[8]), Given(a[9]).get());
        Py_RETURN_NONE;
    });
}

// residual_norm_backward(dy, dh, residual, block, weight, post_weight, gate, scale, eps, dresidual, dblock, dweight, dpost_weight,
//                        dgate, workspace, stream)
PyObject* py_residual_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 16, [&]() -> PyObject* {
        do_norm_backward(maybe(a[0], "dy"), maybe(a[1], "dh"), tensor(a[2], "residual"), maybe(a[3], "block"), tensor(a[4], "weight"),
                         maybe(a[5], "post_weight"), maybe(a[6], "gate"), number(a[7]), number(a[8]), maybe(a[9], "dresidual"),
                         maybe(a[10], "dblock"), maybe(a[11], "dweight"), maybe(a[12], "dpost_weight"), maybe(a[13], "dgate"),
                         maybe(a[14], "workspace"), Given(a[15]).get());
        Py_RETURN_NONE;
    });
}

// linear_cross_entropy(x, w, targets, loss, lse, reduction, workspace, stream)
PyObject* py_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&]() -> PyObject* {
        do_loss(tensor(a[0], "x"), tensor(a[1], "w"), tensor(a[2], "targets"), tensor(a[3], "loss"), maybe(a[4], "lse"), (int)integer(a[5]),
                maybe(a[6], "workspace"), Given(a[7]).get());
        Py_RETURN_NONE;
    });
}

// linear_cross_entropy_backward(dloss, x, w, targets, lse, dx, dw, reduction, workspace, stream)
PyObject* py_loss_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&]() -> PyObject* {
        do_loss_backward(tensor(a[0], "dloss"), tensor(a[1], "x"), tensor(a[2], "w"), tensor(a[3], "targets"), tensor(a[4], "lse"),
                         maybe(a[5], "dx"), maybe(a[6], "dw"), (int)integer(a[7]), maybe(a[8], "workspace"), Given(a[9]).get());
        Py_RETURN_NONE;
    });
}

// apply_embedding(ids, table, scale) -> y
PyObject* py_apply_embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 3, [&]() -> PyObject* {
        const Tensor &ids = tensor(a[0], "ids"), &table = tensor(a[1], "table");
        format_of(table, "table");
        if (table.dim() != 2) refuse("table must be a matrix");
        index_of(ids.contiguous(), ids.numel(), table, "ids");
        on_gpu(table, "table");
        return THPVariable_Wrap(EmbeddingFunction::apply(table, ids, number(a[2])));
    });
}

// apply_palette_embedding(ids, indices, lut, rows, columns, scale, dtype) -> y
PyObject* py_apply_palette_embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject* {
        const Tensor &ids = tensor(a[0], "ids"), &idx = tensor(a[1], "indices"), &lut = tensor(a[2], "lut");
        const int64_t v = integer(a[3]), d = integer(a[4]);
        const double scale = number(a[5]);
        if (!THPDtype_Check(a[6])) refuse("dtype must be a torch type");
        const at::ScalarType type = ((THPDtype*)a[6])->scalar_type;
        if (type != at::kHalf && type != at::kBFloat16) refuse("dtype must be fp16 or bf16, not %s", type_name(type));
        if (lut.requires_grad() && at::GradMode::is_enabled())
            refuse("a palette's table takes no gradient; train the weights through dkm and embedding");
        TORCH_CHECK(!lut._fw_grad(0).defined(), "palette_embedding: forward-mode derivatives are not implemented");
        if (v < 1 || d < 1) refuse("a palette's table has one row and one column at least");
        on_gpu(lut, "lut");
        at::AutoDispatchBelowADInplaceOrView below;
        auto shape = ids.sizes().vec();
        shape.push_back(d);
        Tensor y = at::empty(shape, lut.options().dtype(type));
        do_palette_embedding(ids.contiguous(), idx, lut, v, y.dim() == 2 ? y : y.view({ids.numel(), d}), scale, nullptr);
        return THPVariable_Wrap(y);
    });
}

// apply_norm(residual, weight, block, post_weight, gate, scale, eps) -> y, or (h, y) with a block
PyObject* py_apply_norm(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded(n_args, 7, [&]() -> PyObject* {
        const Tensor &r = tensor(a[0], "residual"), &w = tensor(a[1], "weight");
        const Tensor *u = maybe(a[2], "block"), *post = maybe(a[3], "post_weight"), *gate = maybe(a[4], "gate");
        format_of(r, "residual");
        if (r.dim() < 1) refuse("residual needs a last dimension");
        const int64_t n = r.size(-1);
        like(w, r, "weight");
        if (w.dim() != 1 || w.size(0) != n) refuse("weight must hold %lld elements", (long long)n);
        if (u) {
            like(*u, r, "block");
            if (u->sizes() != r.sizes()) refuse("block must have the residual's shape");
        }
        if (post && (post->dim() != 1 || post->size(0) != n)) refuse("post_weight must hold %lld elements", (long long)n);
        if (post) like(*post, r, "post_weight");
        if (gate && !(gate->dim() == 1 && gate->size(0) == n) && gate->sizes() != r.sizes())
            refuse("gate must hold %lld elements or have the residual's shape", (long long)n);
        if (gate) like(*gate, r, "gate");
        on_gpu(r, "residual");
        auto may = [](const Tensor* t) { return t ? Maybe(*t) : Maybe(); };
        const variable_list o = NormFunction::apply(r, w, may(u), may(post), may(gate), number(a[5]), number(a[6]));
        if (o.size() == 1) return THPVariable_Wrap(o[0]);
        PyObject *h = THPVariable_Wrap(o[0]), *y = THPVariable_Wrap(o[1]);
        PyObject* t = h && y ? PyTuple_Pack(2, h, y) : nullptr;
        Py_XDECREF(h);
        Py_XDECREF(y);
        return t;
    });
}

// apply_loss(x, w, targets, reduction) -> loss
PyObject* py_apply_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject* {
        const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w"), &targets = tensor(a[2], "targets");
        format_of(x, "x");
        if (x.dim() < 1 || w.dim() != 2 || x.size(-1) != w.size(1)) refuse("w must be n x k for x of (..., k)");
        like(w, x, "w");
        bool ok = targets.dim() + 1 == x.dim();
        for (int64_t i = 0; ok && i < targets.dim(); ++i) ok = targets.size(i) == x.size(i);
        if (!ok) refuse("targets must have x's shape without its last dimension");
        index_of(targets.contiguous(), targets.numel(), x, "targets");
        on_gpu(x, "x");
        return THPVariable_Wrap(LossFunction::apply(x, w, targets, integer(a[3])));
    });
}

PyMethodDef methods[] = {
    {"embedding", (PyCFunction)(void*)py_embedding, METH_FASTCALL, nullptr},
    {"palette_embedding", (PyCFunction)(void*)py_palette_embedding, METH_FASTCALL, nullptr},
    {"embedding_backward", (PyCFunction)(void*)py_embedding_backward, METH_FASTCALL, nullptr},
    {"residual_norm", (PyCFunction)(void*)py_residual_norm, METH_FASTCALL, nullptr},
    {"residual_norm_backward", (PyCFunction)(void*)py_residual_norm_backward, METH_FASTCALL, nullptr},
    {"linear_cross_entropy", (PyCFunction)(void*)py_loss, METH_FASTCALL, nullptr},
    {"linear_cross_entropy_backward", (PyCFunction)(void*)py_loss_backward, METH_FASTCALL, nullptr},
    {"apply_embedding", (PyCFunction)(void*)py_apply_embedding, METH_FASTCALL, nullptr},
    {"apply_palette_embedding", (PyCFunction)(void*)py_apply_palette_embedding, METH_FASTCALL, nullptr},
    {"apply_norm", (PyCFunction)(void*)py_apply_norm, METH_FASTCALL, nullptr},
    {"apply_loss", (PyCFunction)(void*)py_apply_loss, METH_FASTCALL, nullptr},
    {"bind", (PyCFunction)(void*)py_bind, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void*)py_linear, METH_FASTCALL, nullptr},
    {"linear_backward", (PyCFunction)(void*)py_linear_backward, METH_FASTCALL, nullptr},
    {"palette_linear", (PyCFunction)(void*)py_palette_linear, METH_FASTCALL, nullptr},
    {"unpalettize", (PyCFunction)(void*)py_unpalettize, METH_FASTCALL, nullptr},
    {"apply_linear", (PyCFunction)(void*)py_apply_linear, METH_FASTCALL, nullptr},
    {"apply_palette_linear", (PyCFunction)(void*)py_apply_palette_linear, METH_FASTCALL, nullptr},
    {"adamw_batch", (PyCFunction)(void*)py_adamw_batch, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_edkm_torch", "Marshalling of libedkm.so's layer and optimizer calls for torch tensors.",
                      -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__edkm_torch() { return PyModule_Create(&module); }
