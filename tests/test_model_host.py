"""Refusals of the operators at a model's ends and between its blocks that need no GPU: the
C ABI rejects bad arguments before any HIP call, and the binding rejects tensors that do not
fit; the sort's plan and the pieces of a vocabulary."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
edkm = pytest.importorskip("paper_2309_00964_amd.edkm",
                           reason="libedkm.so not built (run __graft_entry__.build())")
import torch  # noqa: E402

from paper_2309_00964_amd import function  # noqa: E402

lib = edkm._lib
P = 1 << 40                # never dereferenced: every call below is refused on the host
BIG = 1 << 31
NAN, INF = float("nan"), float("inf")


def embedding(m=4, v=8, d=16, fmt=0, it=1, ids=P, t=P, ldt=16, scale=1.0, y=P, ldy=16):
    return lib.edkm_embedding(m, v, d, fmt, it, ids, t, ldt, scale, y, ldy, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(v=0), dict(d=0), dict(m=BIG), dict(v=BIG), dict(d=BIG), dict(fmt=2), dict(it=2), dict(it=-1),
                                dict(ids=None), dict(t=None), dict(y=None), dict(ldt=15), dict(ldy=15), dict(scale=NAN), dict(scale=INF),
                                dict(v=1 << 21, d=1 << 20, ldt=1 << 20, ldy=1 << 20)])
def test_embedding_argument_errors(kw):
    assert embedding(**kw) == edkm.ERR_ARG


def palette_embedding(m=4, v=8, d=16, bits=3, fmt=0, it=1, ids=P, idx=P, lut=P, scale=1.0, y=P, ldy=16):
    return lib.edkm_palette_embedding(m, v, d, bits, fmt, it, ids, idx, lut, scale, y, ldy, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(v=0), dict(d=0), dict(bits=0), dict(bits=5), dict(fmt=2), dict(it=2), dict(ids=None),
                                dict(idx=None), dict(lut=None), dict(y=None), dict(ldy=15), dict(scale=NAN),
                                dict(v=1 << 17, d=1 << 15, ldy=1 << 15)])
def test_palette_embedding_argument_errors(kw):
    assert palette_embedding(**kw) == edkm.ERR_ARG


def embedding_backward(m=4, v=8, d=16, fmt=0, it=1, ids=P, dy=P, lddy=16, scale=1.0, acc=0, dt=P, lddt=16, ws=P, nws=1 << 20):
    return lib.edkm_embedding_backward(m, v, d, fmt, it, ids, dy, lddy, scale, acc, dt, lddt, ws, nws, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(v=0), dict(d=0), dict(fmt=2), dict(it=2), dict(ids=None), dict(dy=None), dict(dt=None),
                                dict(lddy=15), dict(lddt=15), dict(scale=INF)])
def test_embedding_backward_argument_errors(kw):
    assert embedding_backward(**kw) == edkm.ERR_ARG


def norm(m=4, n=16, fmt=0, r=P, ldr=16, u=P, ldu=16, w=P, post=P, gate=P, ldg=16, rows=0, scale=1.0, eps=1e-6, h=P, ldh=16, y=P, ldy=16):
    return lib.edkm_residual_norm(m, n, fmt, r, ldr, u, ldu, w, post, gate, ldg, rows, scale, eps, h, ldh, y, ldy, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=0), dict(n=edkm.NORM_MAX + 1, ldr=1 << 20, ldu=1 << 20, ldh=1 << 20, ldy=1 << 20), dict(fmt=2),
                                dict(r=None), dict(w=None), dict(y=None), dict(h=None), dict(u=None), dict(u=None, post=None, gate=None),
                                dict(u=None, h=None, post=None), dict(u=None, h=None, gate=None), dict(ldr=15), dict(ldu=15), dict(ldh=15),
                                dict(ldy=15), dict(rows=1, ldg=15), dict(scale=NAN), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF),
                                dict(eps=1e-40)])
def test_norm_argument_errors(kw):
    assert norm(**kw) == edkm.ERR_ARG


def norm_backward(m=4, n=16, fmt=0, dy=P, lddy=16, dh=P, lddh=16, r=P, ldr=16, u=P, ldu=16, w=P, post=P, gate=P, ldg=16, rows=0, scale=1.0,
                  eps=1e-6, dr=P, lddr=16, du=P, lddu=16, dw=P, dp=P, dg=P, ws=P, nws=1 << 20):
    return lib.edkm_residual_norm_backward(m, n, fmt, dy, lddy, dh, lddh, r, ldr, u, ldu, w, post, gate, ldg, rows, scale, eps, dr, lddr, du,
                                           lddu, dw, dp, dg, ws, nws, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=0), dict(fmt=2), dict(r=None), dict(w=None), dict(u=None), dict(post=None), dict(gate=None),
                                dict(dr=None, du=None, dw=None, dp=None, dg=None), dict(lddy=15), dict(lddh=15), dict(ldr=15), dict(ldu=15),
                                dict(lddr=15), dict(lddu=15), dict(rows=1, ldg=15), dict(eps=0.0), dict(scale=INF),
                                dict(u=None, post=None, gate=None, dp=None, dg=None)])
def test_norm_backward_argument_errors(kw):
    assert norm_backward(**kw) == edkm.ERR_ARG


def loss(m=4, n=8, k=16, fmt=0, it=1, red=0, x=P, ldx=16, w=P, ldw=16, t=P, out=P, lse=None, ws=P, nws=1 << 30):
    return lib.edkm_linear_cross_entropy(m, n, k, fmt, it, red, x, ldx, w, ldw, t, out, lse, ws, nws, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=0), dict(k=0), dict(m=BIG), dict(n=BIG), dict(fmt=2), dict(it=2), dict(red=3), dict(red=-1),
                                dict(x=None), dict(w=None), dict(t=None), dict(out=None), dict(ldx=15), dict(ldw=15),
                                dict(m=0, red=1, out=None)])
def test_loss_argument_errors(kw):
    assert loss(**kw) == edkm.ERR_ARG


def loss_backward(m=4, n=8, k=16, fmt=0, it=1, red=0, g=P, x=P, ldx=16, w=P, ldw=16, t=P, lse=P, dx=P, lddx=16, dw=P, ws=P, nws=1 << 30):
    return lib.edkm_linear_cross_entropy_backward(m, n, k, fmt, it, red, g, x, ldx, w, ldw, t, lse, dx, lddx, dw, ws, nws, None)


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=0), dict(k=0), dict(fmt=2), dict(it=2), dict(red=3), dict(g=None), dict(x=None), dict(w=None),
                                dict(t=None), dict(lse=None), dict(dx=None, dw=None), dict(ldx=15), dict(ldw=15), dict(lddx=15)])
def test_loss_backward_argument_errors(kw):
    assert loss_backward(**kw) == edkm.ERR_ARG


def test_workspaces():
    for need, call in ((edkm.embedding_backward_workspace_bytes(4, 8, 16), embedding_backward),
                       (edkm.residual_norm_backward_workspace_bytes(4, 16), norm_backward),
                       (edkm.linear_cross_entropy_workspace_bytes(4, 8, 16), loss),
                       (edkm.linear_cross_entropy_backward_workspace_bytes(4, 8, 16), loss_backward)):
        assert need > 0 and need % 256 == 0
        for kw in (dict(ws=None), dict(ws=P + 128), dict(nws=need - 1)):
            assert call(**kw) == edkm.ERR_WORKSPACE
    assert edkm.embedding_backward_workspace_bytes(0, 8, 16) == 0 == edkm.residual_norm_backward_workspace_bytes(4, 0)
    assert edkm.linear_cross_entropy_workspace_bytes(4, 0, 16) == 0 == edkm.linear_cross_entropy_backward_workspace_bytes(4, 8, 0)
    # the logits are not in it: 16384 x 131072 in 16 bits are 4 GiB
    assert edkm.linear_cross_entropy_workspace_bytes(16384, 131072, 4096) < 1 << 30
    assert edkm.linear_cross_entropy_backward_workspace_bytes(16384, 131072, 4096) < 1 << 30


def test_calls_without_tokens_that_write_nothing():
    assert embedding(m=0, ids=None, y=None) == edkm.OK
    assert palette_embedding(m=0, ids=None, y=None) == edkm.OK
    assert embedding_backward(m=0, ids=None, dy=None, acc=1, ws=None, nws=0) == edkm.OK
    assert norm(m=0, r=None, u=None, h=None, y=None) == edkm.OK
    assert norm_backward(m=0, dy=None, dh=None, r=None, u=None, dr=None, du=None, dw=None, dp=None, dg=None, ws=None, nws=0) == edkm.OK
    assert loss(m=0, x=None, t=None, out=None) == edkm.OK
    assert loss_backward(m=0, g=None, x=None, t=None, lse=None, dx=None, dw=None, ws=None, nws=0) == edkm.OK


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "edkm.h")).read()
    assert {k.lower(): int(v) for k, v in re.findall(r"\bEDKM_REDUCE_([A-Z]+)\s*=\s*(\d+)", text)} == edkm.REDUCTIONS
    assert dict(re.findall(r"\bEDKM_INDEX_([A-Z0-9]+)\s*=\s*(\d+)", text)) == {"INT32": str(edkm.INDEX_INT32), "INT64": str(edkm.INDEX_INT64)}
    assert int(re.search(r"#define EDKM_NORM_MAX (\d+)", text).group(1)) == edkm.NORM_MAX


def h(*shape, dtype=torch.float16, device="cpu"):
    """Host memory: the last refusal is that it is no device tensor; "meta" stands for another device."""
    return torch.zeros(shape, dtype=dtype, device=device)


IDS, F32 = torch.zeros(4, dtype=torch.int64), torch.float32


@pytest.mark.parametrize("call,what", [
    (lambda: edkm.embedding(IDS, h(8, 16), h(4, 15)), "y must be"),
    (lambda: edkm.embedding(IDS, h(8, 16), h(3, 16)), "y must be"),
    (lambda: edkm.embedding(IDS, h(8, 16), h(4, 16, dtype=torch.bfloat16)), "y must have"),
    (lambda: edkm.embedding(IDS.float(), h(8, 16), h(4, 16)), "ids must be int32"),
    (lambda: edkm.embedding(IDS.to("meta"), h(8, 16), h(4, 16)), "ids must be on"),
    (lambda: edkm.embedding(torch.zeros(8, dtype=torch.int64)[::2], h(8, 16), h(4, 16)), "contiguous"),
    (lambda: edkm.embedding(IDS, h(8, 16, dtype=F32), h(4, 16, dtype=F32)), "fp16 or bf16"),
    (lambda: edkm.embedding(IDS, h(8, 16), h(4, 16)), "device tensor"),
    (lambda: edkm.embedding(IDS, h(16, 8).t(), h(4, 16)), "contiguous rows"),
    (lambda: edkm.embedding_backward(IDS, h(4, 16), h(8, 15)), "dy must be"),
    (lambda: edkm.embedding_backward(IDS, h(4, 16), h(8, 16)), "device tensor"),
    (lambda: edkm.palette_embedding(IDS, h(48, dtype=torch.uint8), h(8, dtype=F32), 8, h(4, 17)), "indices must be"),
    (lambda: edkm.palette_embedding(IDS, h(48, dtype=torch.uint8), h(7, dtype=F32), 8, h(4, 16)), "lut must hold"),
    (lambda: edkm.palette_embedding(IDS, h(48, dtype=torch.uint8), h(8, dtype=F32), 0, h(4, 16)), "one row"),
    (lambda: edkm.palette_embedding(IDS, h(48, dtype=torch.uint8), h(8, dtype=F32), 8, h(4, 16)), "device tensor"),
    (lambda: edkm.residual_norm(h(4, 16), h(15), h(4, 16)), "weight must hold"),
    (lambda: edkm.residual_norm(h(4, 16), h(16), h(4, 16), h(4, 16)), "belong to a block"),
    (lambda: edkm.residual_norm(h(4, 16), h(16), h(4, 16), None, h(4, 16)), "needs h"),
    (lambda: edkm.residual_norm(h(4, 16), h(16), h(4, 16), h(4, 16), h(4, 16), None, h(4, 15)), "gate must be"),
    (lambda: edkm.residual_norm(h(4, 16), h(16), h(4, 16), h(4, 16), h(4, 16), None, h(15)), "gate must hold"),
    (lambda: edkm.residual_norm(h(4, 16), h(16), h(4, 16)), "device tensor"),
    (lambda: edkm.residual_norm_backward(None, None, h(4, 16), h(16), dgate=h(16)), "not given"),
    (lambda: edkm.residual_norm_backward(None, None, h(4, 16), h(16), dblock=h(4, 16)), "belong to a block"),
    (lambda: edkm.residual_norm_backward(None, None, h(4, 16), h(16), dresidual=h(4, 16)), "device tensor"),
    (lambda: edkm.linear_cross_entropy(h(4, 16), h(8, 15), IDS, h(4, dtype=F32)), "w must be"),
    (lambda: edkm.linear_cross_entropy(h(4, 16), h(8, 16), IDS[:3], h(4, dtype=F32)), "targets must hold"),
    (lambda: edkm.linear_cross_entropy(h(4, 16), h(8, 16), IDS, h(4)), "loss must hold"),
    (lambda: edkm.linear_cross_entropy(h(4, 16), h(8, 16), IDS, h(4, dtype=F32), None, "sum"), "loss must hold 1"),
    (lambda: edkm.linear_cross_entropy(h(4, 16), h(8, 16), IDS, h(4, dtype=F32), None, "median"), "reduction"),
    (lambda: edkm.linear_cross_entropy(h(4, 16), h(8, 16), IDS, h(4, dtype=F32)), "device tensor"),
    (lambda: edkm.linear_cross_entropy_backward(h(1, dtype=F32), h(4, 16), h(8, 16), IDS, h(4, dtype=F32), h(4, 16)), "dloss must hold"),
    (lambda: edkm.linear_cross_entropy_backward(h(4, dtype=F32), h(4, 16), h(8, 16), IDS, h(3, dtype=F32), h(4, 16)), "lse must hold"),
    (lambda: edkm.linear_cross_entropy_backward(h(4, dtype=F32), h(4, 16), h(8, 16), IDS, h(4, dtype=F32), h(4, 16), h(7, 16)), "dw must hold"),
    (lambda: function.embedding(IDS, h(8)), "matrix"),
    (lambda: function.embedding(IDS.double(), h(8, 16)), "int32 or int64"),
    (lambda: function.embedding(IDS, h(8, 16)), "device tensor"),
    (lambda: function.palette_embedding(IDS, h(48, dtype=torch.uint8), h(8, dtype=F32), 8, 16, dtype=F32), "dtype must be"),
    (lambda: function.palette_embedding(IDS, h(48, dtype=torch.uint8), h(8, dtype=F32).requires_grad_(), 8, 16), "no gradient"),
    (lambda: function.palette_embedding(IDS, h(48, dtype=torch.uint8), h(8, dtype=F32), 8, 16), "device tensor"),
    (lambda: function.rms_norm(h(2, 3, 16), h(15)), "weight must hold"),
    (lambda: function.rms_norm(h(2, 3, 16), h(16)), "device tensor"),
    (lambda: function.residual_norm(h(2, 3, 16), h(3, 2, 16), h(16)), "block must have"),
    (lambda: function.residual_norm(h(2, 3, 16), h(2, 3, 16), h(16), h(15)), "post_weight must hold"),
    (lambda: function.residual_norm(h(2, 3, 16), h(2, 3, 16), h(16), None, h(2, 1, 16)), "gate must hold"),
    (lambda: function.residual_norm(h(2, 3, 16), h(2, 3, 16), h(16), None, h(16, dtype=F32)), "gate must have"),
    (lambda: function.linear_cross_entropy(h(2, 2, 16), h(8, 16), IDS), "targets must have"),
    (lambda: function.linear_cross_entropy(h(4, 16), h(8, 17), IDS), "n x k"),
    (lambda: function.linear_cross_entropy(h(4, 16), h(8, 16), IDS, "max"), "reduction"),
    (lambda: function.linear_cross_entropy(h(4, 16), h(8, 16), IDS), "device tensor"),
])
def test_binding_refuses_what_does_not_fit(call, what):
    with pytest.raises(ValueError, match=what):
        call()


def test_embedding_is_bounded_by_its_matrices():
    """m x d and v x d are the embedding's matrices; there is none of m x v."""
    m, v = (1 << 22) + 1, 1 << 18
    assert edkm.embedding_backward_workspace_bytes(m, v, 8) > 0
    assert embedding_backward(m=m, v=v, d=8, lddy=8, lddt=8, ws=None) == edkm.ERR_WORKSPACE
    for kw in (dict(m=1 << 21, v=1, d=1 << 20), dict(m=1, v=1 << 21, d=1 << 20)):
        assert edkm.embedding_backward_workspace_bytes(**kw) == 0
        assert embedding(**kw, ldt=1 << 20, ldy=1 << 20) == edkm.ERR_ARG
        assert embedding_backward(**kw, lddy=1 << 20, lddt=1 << 20) == edkm.ERR_ARG
    assert palette_embedding(m=1 << 21, v=1, d=1 << 20, ldy=1 << 20) == edkm.ERR_ARG
