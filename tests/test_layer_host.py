"""Refusals of the layer and optimizer operators that need no GPU: the C ABI rejects bad
arguments before any HIP call, and the binding rejects tensors that do not fit."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
edkm = pytest.importorskip("paper_2309_00964_amd.edkm",
                           reason="libedkm.so not built (run __graft_entry__.build())")
import torch  # noqa: E402

lib = edkm._lib
P = 1 << 40                # never dereferenced: every call below is refused on the host
BIG = 1 << 31


def linear(m=4, n=8, k=16, fmt=0, act=0, x=P, ldx=16, w=P, ldw=16, bias=None, res=None, ldr=8, y=P, ldy=8, z=None, ws=None,
           nws=0):
    return lib.edkm_linear(m, n, k, fmt, act, x, ldx, w, ldw, bias, res, ldr, y, ldy, z, ws, nws, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=0), dict(k=0), dict(m=BIG), dict(n=BIG), dict(k=BIG), dict(fmt=2), dict(fmt=-1),
                                dict(act=4), dict(act=-1), dict(x=None), dict(w=None), dict(y=None), dict(ldx=15), dict(ldw=15),
                                dict(ldy=7), dict(res=P, ldr=7), dict(ldx=1 << 41)])
def test_linear_argument_errors(kw):
    assert linear(**kw) == edkm.ERR_ARG


def backward(m=4, n=8, k=16, fmt=0, act=0, dy=P, lddy=8, z=None, x=P, ldx=16, w=P, ldw=16, dx=P, lddx=16, dw=P, db=P, ws=P,
             nws=1 << 30):
    return lib.edkm_linear_backward(m, n, k, fmt, act, dy, lddy, z, x, ldx, w, ldw, dx, lddx, dw, db, ws, nws, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=0), dict(k=0), dict(fmt=2), dict(act=4), dict(dx=None, dw=None, db=None),
                                dict(dy=None), dict(act=1), dict(x=None), dict(w=None), dict(lddy=7), dict(lddx=15), dict(ldx=15),
                                dict(ldw=15)])
def test_linear_backward_argument_errors(kw):
    assert backward(**kw) == edkm.ERR_ARG


def test_workspaces():
    need = edkm.linear_backward_workspace_bytes(400, 800, 64, "silu")
    assert need >= 400 * 800 * 2
    assert edkm.linear_backward_workspace_bytes(400, 0, 64) == 0
    a = dict(m=400, n=800, k=64, act=3, z=P, lddy=800, ldx=64, ldw=64, lddx=64)
    assert backward(ws=None, **a) == edkm.ERR_WORKSPACE
    assert backward(nws=need - 1, **a) == edkm.ERR_WORKSPACE
    assert backward(ws=P + 16, **a) == edkm.ERR_WORKSPACE
    for m, n, k in ((1, 64, 4096), (300, 4096, 4096), (5000, 256, 256)):
        need = edkm.linear_workspace_bytes(m, n, k)
        assert need % 256 == 0
        if need:
            assert linear(m=m, n=n, k=k, ldx=k, ldw=k, ldy=n, ws=P, nws=need - 1) == edkm.ERR_WORKSPACE
        assert edkm.palette_linear_workspace_bytes(m, n, k, 3) % 256 == 0


def palette(m=4, n=8, k=16, bits=3, fmt=0, act=0, x=P, ldx=16, idx=P, lut=P, bias=None, res=None, ldr=8, y=P, ldy=8, z=None,
            ws=None, nws=0):
    return lib.edkm_palette_linear(m, n, k, bits, fmt, act, x, ldx, idx, lut, bias, res, ldr, y, ldy, z, ws, nws, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=0), dict(k=0), dict(bits=0), dict(bits=5), dict(fmt=2), dict(act=4), dict(x=None),
                                dict(idx=None), dict(lut=None), dict(y=None), dict(ldx=15), dict(ldy=7), dict(res=P, ldr=7),
                                dict(n=1 << 17, k=1 << 15, ldx=1 << 15, ldy=1 << 17)])
def test_palette_linear_argument_errors(kw):
    assert palette(**kw) == edkm.ERR_ARG


def test_unpalettize_argument_errors():
    f = lib.edkm_unpalettize
    assert f(None, 10, 3, 0, P, P, None) == edkm.ERR_ARG
    assert f(P, 10, 3, 0, None, P, None) == edkm.ERR_ARG
    assert f(P, 10, 3, 0, P, None, None) == edkm.ERR_ARG
    assert f(P, 0, 3, 0, P, P, None) == edkm.ERR_ARG
    assert f(P, 1 << 32, 3, 0, P, P, None) == edkm.ERR_ARG
    for bits, fmt in ((0, 0), (5, 0), (3, 2)):
        assert f(P, 10, bits, fmt, P, P, None) == edkm.ERR_ARG


def adamw(sizes=(100, 50), pt=0, gt=0, bits=32, p=(P, 2 * P), w=None, g=(P, P), m=(3 * P, 4 * P), v=(5 * P, 6 * P), ms=None, vs=None,
          step=P, lr_dev=None, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, count=None):
    arr = lambda x: None if x is None else (ctypes.c_void_p * len(x))(*x)  # noqa: E731
    return lib.edkm_adamw_batch(len(sizes) if count is None else count, (ctypes.c_uint64 * len(sizes))(*sizes), pt, gt, bits, arr(p),
                                arr(w), arr(g), arr(m), arr(v), arr(ms), arr(vs), step, lr_dev, lr, b1, b2, eps, wd, 0, None)


NAN = float("nan")


@pytest.mark.parametrize("kw", [dict(count=0), dict(sizes=(1 << 32, 5)), dict(pt=3), dict(pt=-1), dict(gt=1), dict(pt=2, gt=0),
                                dict(bits=16), dict(bits=8), dict(bits=8, ms=(P, P)), dict(pt=2, gt=2, w=(P, P)), dict(step=None),
                                dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(p=(P, None)), dict(m=(None, P)),
                                dict(bits=8, ms=(P, None), vs=(P, P)), dict(lr=NAN), dict(lr=-1.0), dict(b1=1.0), dict(b1=NAN),
                                dict(b2=-0.1), dict(eps=NAN), dict(eps=-1.0), dict(wd=-1.0), dict(wd=NAN), dict(lr=float("inf")),
                                dict(p=(P, P)), dict(p=(P, P + 198)), dict(m=(3 * P, 3 * P + 396)), dict(v=(5 * P + 4, 5 * P))])
def test_adamw_argument_errors(kw):
    assert adamw(**kw) == edkm.ERR_ARG


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "edkm.h")).read()
    acts = {k.lower(): int(v) for k, v in re.findall(r"\bEDKM_ACT_([A-Z]+)\s*=\s*(\d+)", text)}
    assert acts == edkm.ACTIVATIONS
    types = {k: int(v) for k, v in re.findall(r"\bEDKM_TYPE_([A-Z0-9]+)\s*=\s*(\d+)", text)}
    assert types == {k: getattr(edkm, "TYPE_" + k) for k in ("FP16", "BF16", "FP32")}
    assert int(re.search(r"#define EDKM_STATE_BLOCK (\d+)", text).group(1)) == edkm.STATE_BLOCK


def h(*shape, dtype=torch.float16, stride=None, device="cpu"):
    """A tensor of a shape, type and stride (host memory: the last refusal is that it is no
    device tensor; one on "meta" stands for another device)."""
    if stride is None:
        return torch.zeros(shape, dtype=dtype, device=device)
    return torch.zeros(1 << 10, dtype=dtype, device=device).as_strided(shape, stride)


def test_binding_refuses_matrices_that_do_not_fit():
    x, w, y = h(4, 16), h(8, 16), h(4, 8)
    cases = [
        (lambda: edkm.linear(h(4, 16, dtype=torch.float32), w, y), "x must be"),
        (lambda: edkm.linear(x, h(8, 15), y), "w must be 8 x 16"),
        (lambda: edkm.linear(x, w, h(4, 9)), "y must be 4 x 8"),
        (lambda: edkm.linear(x, w, h(4, 8, dtype=torch.bfloat16)), "y must have the type"),
        (lambda: edkm.linear(x, w, h(4, 8, device="meta")), "y must have the type and device"),
        (lambda: edkm.linear(h(4, 16, stride=(1, 4)), w, y), "x must have contiguous rows"),
        (lambda: edkm.linear(h(4, 16, stride=(0, 1)), w, y), "x must have contiguous rows"),
        (lambda: edkm.linear(x, w, y, h(7)), "bias must hold 8"),
        (lambda: edkm.linear(x, w, y, None, h(4, 7)), "residual must be"),
        (lambda: edkm.linear(x, w, y, None, None, "tanh"), "activation"),
        (lambda: edkm.linear(x, w, y, z_out=h(4, 9)), "z_out"),
        (lambda: edkm.linear_backward(y, None, w, dw=h(8, 16)), "dw needs x"),
        (lambda: edkm.linear_backward(y, x, None, dx=h(4, 16)), "dx needs w"),
        (lambda: edkm.linear_backward(y, x, w, dx=h(4, 16), activation="silu"), "needs z"),
        (lambda: edkm.linear_backward(y, x, w, dw=h(8, 15)), "dw must hold"),
        (lambda: edkm.palette_linear(x, h(47, dtype=torch.uint8), h(8, dtype=torch.float32), y), "indices must be 48"),
        (lambda: edkm.palette_linear(x, h(48, dtype=torch.uint8), h(8), y), "lut must hold"),
        (lambda: edkm.palette_linear(x, h(48, dtype=torch.uint8), h(32, dtype=torch.float32), y), "lut must hold"),
        (lambda: edkm.unpalettize(h(48, dtype=torch.uint8, device="meta"), h(8, dtype=torch.float32), h(128)), "must be on cpu"),
        (lambda: edkm.unpalettize(h(48, dtype=torch.uint8), h(8, dtype=torch.float32), h(129)), "indices must be 49"),
        (lambda: edkm.unpalettize(h(48, dtype=torch.uint8), h(8, dtype=torch.float32), h(128)), "device tensor"),
        (lambda: edkm.linear(x, w, y), "device tensor"),
        (lambda: edkm.linear_backward(y, x, w, dx=h(4, 16)), "device tensor"),
        (lambda: edkm.palette_linear(x, h(48, dtype=torch.uint8), h(8, dtype=torch.float32), y), "device tensor"),
        (lambda: edkm.linear(None, w, y), "x must be a tensor"),
    ]
    for call, what in cases:
        with pytest.raises(ValueError, match=what):
            call()


def test_binding_refuses_optimizer_lists_that_do_not_fit():
    f32 = torch.float32
    p, g, q = [h(300), h(5)], [h(300), h(5)], h(204)
    m, v, step = [h(300, dtype=f32), h(5, dtype=f32)], [h(300, dtype=f32), h(5, dtype=f32)], h(1, dtype=torch.int32)
    e8 = [h(300, dtype=torch.float8_e4m3fn), h(5, dtype=torch.float8_e4m3fn)]
    e5 = [h(300, dtype=torch.float8_e5m2), h(5, dtype=torch.float8_e5m2)]
    s2, s1 = [h(2, dtype=f32), h(1, dtype=f32)], [h(1, dtype=f32), h(1, dtype=f32)]
    cases = [
        (lambda: edkm.adamw_batch(p, g[:1], m, v, step, 1e-3), "grads has 1 entries"),
        (lambda: edkm.adamw_batch(p, [h(300), h(4)], m, v, step, 1e-3), "grads"),
        (lambda: edkm.adamw_batch(p, [h(300, dtype=torch.bfloat16)] * 2, m, v, step, 1e-3), "grads"),
        (lambda: edkm.adamw_batch(p, g, m, v, step, 1e-3), "device tensors"),
        (lambda: edkm.adamw_batch([q[:200], q[199:]], g, m, v, step, 1e-3), "overlap"),
        (lambda: edkm.adamw_batch([p[1], p[1]], g, m, v, step, 1e-3), "twice"),
        (lambda: edkm.adamw_batch(p, g, e8, v, step, 1e-3), "exp_avgs"),
        (lambda: edkm.adamw_batch(p, g, e8, e5, step, 1e-3, m_scales=s2), "m_scales and v_scales"),
        (lambda: edkm.adamw_batch(p, g, e8, e5, step, 1e-3, m_scales=s1, v_scales=s2), "m_scales"),
        (lambda: edkm.adamw_batch(p, g, e8, e8, step, 1e-3, m_scales=s2, v_scales=s2), "exp_avg_sqs"),
        (lambda: edkm.adamw_batch(p, g, m, v, h(1, dtype=torch.int64), 1e-3), "step"),
        (lambda: edkm.adamw_batch(p, g, m, v, step, torch.zeros(1, dtype=torch.float64)), "lr"),
        (lambda: edkm.adamw_batch(m, g, m, v, step, 1e-3), "grads"),
        (lambda: edkm.adamw_batch(m, m, m, v, step, 1e-3, masters=m), "take no masters"),
        (lambda: edkm.adamw_batch([h(4, 4, stride=(1, 4))], [h(16)], [h(16, dtype=f32)], [h(16, dtype=f32)], step, 1e-3), "contiguous"),
    ]
    for call, what in cases:
        with pytest.raises((ValueError, edkm.EdkmError), match=what):
            call()


def test_function_refusals():
    from paper_2309_00964_amd import function
    x, w = torch.zeros(2, 3, 16, dtype=torch.float16), torch.zeros(8, 16, dtype=torch.float16)
    lut = torch.zeros(8)
    for call, what in [
        (lambda: function.linear(x, w), "device tensor"),
        (lambda: function.linear(x, w[:, :15]), "w must be n x k"),
        (lambda: function.linear(x, w, torch.zeros(7)), "bias must hold 8"),
        (lambda: function.linear(x, w, None, torch.zeros(2, 4, 8)), "residual must have"),
        (lambda: function.palette_linear(x, torch.zeros(48, dtype=torch.uint8), lut, 8), "device tensor"),
        (lambda: function.palette_linear(x, torch.zeros(48, dtype=torch.uint8), lut, 8, torch.zeros(9)), "bias must hold 8"),
        (lambda: function.palette_linear(x, torch.zeros(48, dtype=torch.uint8), lut.requires_grad_(True), 8), "no gradient"),
    ]:
        with pytest.raises(ValueError, match=what):
            call()


def test_optimizer_refusals():
    from paper_2309_00964_amd.optim import AdamW
    p = torch.nn.Parameter(torch.zeros(4))
    for kw, what in ((dict(state_bits=16), "state_bits"), (dict(lr=-1.0), "lr"), (dict(lr=float("nan")), "lr"), (dict(betas=(1.0, 0.9)), "betas"),
                     (dict(eps=-1.0), "eps"), (dict(weight_decay=float("inf")), "weight_decay"),
                     (dict(lr=torch.zeros(2)), "tensor lr")):
        with pytest.raises(ValueError, match=what):
            AdamW([p], **kw)
    with pytest.raises(ValueError, match="float64"):
        AdamW([torch.nn.Parameter(torch.zeros(4, dtype=torch.float64))])
    opt = AdamW([p])
    opt.step()                       # no gradient: nothing to do
    p.grad = torch.zeros(4)
    with pytest.raises(ValueError, match="GPU tensors"):
        opt.step()
    q = torch.nn.Parameter(torch.zeros(4, dtype=torch.float16))
    q.grad = torch.zeros(4, dtype=torch.float16)
    with pytest.raises(ValueError, match="GPU tensors"):
        AdamW([q]).step()


@pytest.mark.parametrize("which", ["x", "bias", "residual", "lut"])
@pytest.mark.parametrize("grad", [False, True])
def test_palette_linear_refuses_forward_derivatives(which, grad):
    """A tangent is never dropped, which would count as a zero derivative."""
    from torch.autograd import forward_ad
    from paper_2309_00964_amd import function
    t = dict(x=h(4, 16), bias=h(8), residual=h(4, 8), lut=h(8, dtype=torch.float32))
    other = "bias" if which == "x" else "x"
    with forward_ad.dual_level():
        t[which] = forward_ad.make_dual(t[which], torch.ones_like(t[which]))
        t[other] = t[other].requires_grad_(grad)
        for mode in (torch.enable_grad, torch.no_grad):
            with mode(), pytest.raises(RuntimeError, match="forward-mode derivatives"):
                function.palette_linear(t["x"], h(48, dtype=torch.uint8), t["lut"], 8, t["bias"], t["residual"])


def test_backward_of_no_tokens_that_writes_nothing():
    """An empty dx (a null pointer, or any) and no other gradient: nothing to do, no workspace."""
    for dx in (None, P):
        for act in (0, 3):
            assert backward(m=0, act=act, dy=None, x=None, dx=dx, dw=None, db=None, ws=None, nws=0) == edkm.OK
    assert backward(m=0, n=0, dx=None, dw=None, db=None) == edkm.ERR_ARG
    assert backward(m=0, dw=None, db=None, w=None) == edkm.ERR_ARG


E8 = dict(bits=8, ms=(7 * P, 8 * P), vs=(9 * P, 10 * P), sizes=(1000, 500))


@pytest.mark.parametrize("kw", [dict(w=(7 * P, 7 * P)), dict(w=(7 * P, 7 * P + 396)), dict(w=(7 * P + 196, 7 * P)),
                                dict(E8, ms=(7 * P, 7 * P)), dict(E8, ms=(7 * P, 7 * P + 12)), dict(E8, vs=(9 * P + 4, 9 * P)),
                                dict(v=(4 * P, 6 * P)), dict(w=(P, 7 * P)), dict(w=(None, P)), dict(E8, ms=(7 * P, 9 * P + 12)),
                                dict(m=(3 * P, 4 * P), v=(3 * P + 400 - 4, 6 * P))])
def test_adamw_refuses_arrays_that_overlap(kw):
    """Masters and block scales too, and arrays of two kinds: all that one launch writes."""
    assert adamw(**kw) == edkm.ERR_ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="the pointers are none: no launch may come of them")
@pytest.mark.parametrize("kw", [dict(w=(7 * P, 7 * P + 400)), E8, dict(E8, ms=(7 * P, 7 * P + 16)), dict(E8, vs=(9 * P + 8, 9 * P)),
                                dict(w=(7 * P + 200, 7 * P)), dict(w=(None, None)), dict(g=(P, P))])
def test_adamw_accepts_neighbouring_arrays(kw):
    """Past the checks, where without a GPU the launch fails."""
    assert adamw(**kw) == edkm.ERR_HIP


PARTS = r'''
#include "edkm_launch.h"
#include <cstdio>
int main() {
    unsigned long long groups;
    unsigned threads, fail;
    while (std::scanf("%llu %u %u", &groups, &threads, &fail) == 3) {
        unsigned calls = 0;
        int s = edkm::in_parts(groups, threads, 0, [&](uint32_t first, uint32_t n) {
            std::printf("%u %u ", first, n);
            return ++calls == fail ? 7 : 0;
        });
        std::printf("= %d\n", s);
    }
}
'''


def test_parts_of_a_large_grid(tmp_path):
    """Every workgroup once and in order, fewer than 2^32 threads a launch, parts that start on
    a multiple of eight, and nothing more after a part that fails."""
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    (tmp_path / "parts.cpp").write_text(PARTS)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2309_00964_amd", "csrc"), "-o",
                           str(tmp_path / "parts"), str(tmp_path / "parts.cpp")])
    cases = [(g, t, f) for t in (64, 128, 256, 512, 1024) for g in (1, 7, (1 << 32) // t - 1, (1 << 32) // t, (1 << 31) // 16, (1 << 32) - 1)
             for f in (0, 1, 2)]
    text = "".join("%d %d %d\n" % c for c in cases)
    lines = subprocess.run([str(tmp_path / "parts")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(lines) == len(cases)
    for (groups, threads, fail), line in zip(cases, lines):
        parts, status = line.split("=")
        vals = [int(v) for v in parts.split()]
        at = 0
        for first, n in zip(vals[::2], vals[1::2]):
            assert first == at and first % 8 == 0 and n >= 1 and n * threads < 1 << 32
            at += n
        assert at <= groups and (int(status) == 7) == (fail > 0 and len(vals) // 2 == fail)
        assert at == groups or int(status) == 7


@pytest.mark.parametrize("kw,what", [(dict(state_bits=16), "state_bits"), (dict(lr=-1.0), "lr"), (dict(lr=float("nan")), "lr"),
                                     (dict(lr=torch.zeros(2)), "tensor lr"), (dict(lr=torch.zeros(1, dtype=torch.float64)), "tensor lr"),
                                     (dict(betas=(0.9, 1.0)), "betas"), (dict(eps=float("inf")), "eps"), (dict(weight_decay=-1.0), "weight_decay"),
                                     (dict(params=[torch.nn.Parameter(torch.zeros(4, dtype=torch.float64))]), "float64")])
def test_optimizer_checks_a_groups_own_options(kw, what):
    from paper_2309_00964_amd.optim import AdamW
    group = lambda: dict(dict(params=[torch.nn.Parameter(torch.zeros(4))]), **kw)  # noqa: E731
    with pytest.raises(ValueError, match=what):
        AdamW([group()])
    opt = AdamW([torch.nn.Parameter(torch.zeros(3))])
    with pytest.raises(ValueError, match=what):
        opt.add_param_group(group())
    assert len(opt.param_groups) == 1          # the refused group is not kept
    opt.add_param_group(dict(params=[torch.nn.Parameter(torch.zeros(4))], lr=torch.zeros(1), state_bits=8))
    assert len(opt.param_groups) == 2


@pytest.mark.parametrize("m,n,k,bits", [(65, 4096, 4096, 3), (128, 4096, 4096, 3), (300, 4096, 4096, 4), (1024, 4096, 4096, 1)])
def test_palette_workspace_holds_no_weights_that_are_decoded_on_the_way(m, n, k, bits):
    """An aligned copy of x and a split's sums at most; the weights where they are decoded first."""
    assert edkm.palette_linear_workspace_bytes(m, n, k, bits) <= 2 * m * k + edkm.linear_workspace_bytes(m, n, k)
    assert edkm.palette_linear_workspace_bytes(4096, n, k, bits) >= 2 * n * k
    assert edkm.palette_linear_workspace_bytes(m, n, k + 1, bits) >= 2 * n * (k + 1)
