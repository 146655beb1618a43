"""Embedding, norms between blocks and the cross entropy of a product against plain 64-bit
forms: every type, sizes around the ends of tiles and chunks, strided and unaligned rows,
buffers whose surroundings are NaN, tokens that stand for none, empty batches."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_util as L                                             # noqa: E402
import model_util as M                                             # noqa: E402
from oracle import palette as pal                                  # noqa: E402
from paper_2309_00964_amd import edkm, function                    # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"


def say(*a):
    print("[gpu-case]", *a, flush=True)
    sys.stdout.flush()


def randn(seed, *shape, dtype, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def tokens(seed, m, v, kind="log", dtype=torch.int64):
    """Tokens of a table of v rows: frequent ones ("log"), all alike ("one"), each once or
    nearly ("flat"), none ("none"); a tenth stand for none, in each of the ways they can."""
    rng = np.random.default_rng(seed)
    t = {"log": lambda: np.minimum((np.exp(rng.random(m) * np.log(v + 1)) - 1).astype(np.int64), v - 1),
         "one": lambda: np.full(m, v // 2), "flat": lambda: rng.integers(0, v, m), "none": lambda: np.full(m, -1)}[kind]()
    if kind != "one":
        out = rng.random(m) < 0.1
        ways = [-1, -100, v, 2 ** 31 - 1, -2 ** 31] + ([2 ** 32, 2 ** 63 - 1, -2 ** 63, 2 ** 32 * 5] if dtype == torch.int64 else [])
        t[out] = np.array(ways, dtype=np.int64)[rng.integers(0, len(ways), int(out.sum()))]
    return torch.from_numpy(t).to(dtype).to(DEV)


def inside(t, lead=1, gap=0):
    """The same matrix as a view of a NaN-filled buffer: `lead` elements and one row before
    it, `gap` elements between its rows, a row after it."""
    r, c = t.shape
    buf = torch.full((lead + (r + 2) * (c + gap),), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[lead + c + gap:][: r * (c + gap)].view(r, c + gap)[:, :c]
    v.copy_(t)
    return buf, v


# ---------------------------------------------------------------------------
# embedding

EMBED = [(1, 1, 1, "flat"), (1, 300, 64, "log"), (5, 7, 3, "log"), (16, 40, 8, "one"), (17, 40, 24, "one"), (100, 33, 129, "log"),
         (257, 1000, 77, "flat"), (1001, 64, 200, "log"), (333, 50, 2056, "one"), (8192, 129, 40, "log"), (8193, 129, 40, "log"),
         (20000, 70000, 16, "log"), (9000, 1023, 9, "one"), (40000, 1024, 33, "log"), (12, 5, 4099, "none"), (70000, 300000, 2, "flat")]


@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
@pytest.mark.parametrize("m,v,d,kind", EMBED)
def test_embedding(fmt, m, v, d, kind):
    dt, itype = L.DT[fmt], torch.int32 if m % 2 else torch.int64
    say("embedding", fmt, m, v, d, kind)
    ids, table, dy = tokens(m, m, v, kind, itype), randn(1, v, d, dtype=dt), randn(2, m, d, dtype=dt)
    for scale in (1.0, -0.37):
        y = torch.empty(m, d, dtype=dt, device=DEV)
        edkm.embedding(ids, table, y, scale)
        L.assert_within(y, *M.embedding(ids, table, scale), "y")
        g = torch.full((v, d), float("nan"), dtype=dt, device=DEV)
        edkm.embedding_backward(ids, dy, g, scale)
        ref, tol = M.embedding_grad(ids, dy, v, scale)
        L.assert_within(g, ref, tol, "dtable")
        named = ids[(ids >= 0) & (ids < v)].long().unique()
        rest = torch.ones(v, dtype=torch.bool, device=DEV)
        rest[named] = False
        assert not bool(g[rest].any())
        again = torch.empty_like(g)
        edkm.embedding_backward(ids, dy, again, scale)
        assert torch.equal(g, again)
        old = randn(3, v, d, dtype=dt)
        more = old.clone()
        more[rest] = float("nan")
        edkm.embedding_backward(ids, dy, more, scale, accumulate=True)
        ref, tol = M.embedding_grad(ids, dy, v, scale, old)
        L.assert_within(more[named], ref[named], tol[named], "accumulated")
        assert bool(more[rest].isnan().all())


@pytest.mark.parametrize("m,v,d,kind", [(131073, 4, 8, "log"), (60000, 2, 65, "flat"), (50001, 3, 130, "flat"), (34000, 5, 257, "one"),
                                        (33000, 1, 520, "flat"), (20000, 3, 1100, "log")])
def test_embedding_rows_of_many_chunks(m, v, d, kind):
    """Rows whose tokens fill hundreds of chunks, at each number of threads that join them."""
    dt = torch.bfloat16
    say("embedding chunks", m, v, d, kind)
    ids, dy, old = tokens(m, m, v, kind), randn(2, m, d, dtype=dt), randn(3, v, d, dtype=dt)
    for accumulate in (False, True):
        g = old.clone()
        edkm.embedding_backward(ids, dy, g, 0.5, accumulate)
        ref, tol = M.embedding_grad(ids, dy, v, 0.5, *([old] if accumulate else []))
        named = ids[(ids >= 0) & (ids < v)].long().unique() if accumulate else slice(None)
        L.assert_within(g[named], ref[named], tol[named], "dtable")


@pytest.mark.parametrize("d,lead,gap", [(64, 1, 3), (64, 8, 8), (77, 3, 0), (129, 8, 7)])
def test_embedding_views_in_nan_buffers(d, lead, gap):
    dt, m, v = torch.bfloat16, 200, 60
    say("embedding views", d, lead, gap)
    ids = tokens(5, m, v)
    table, dy = randn(1, v, d, dtype=dt), randn(2, m, d, dtype=dt)
    _, tv = inside(table, lead, gap)
    _, dyv = inside(dy, lead, gap)
    ybuf, yv = inside(torch.zeros_like(dy), lead, gap)
    gbuf, gv = inside(torch.zeros_like(table), lead, gap)
    edkm.embedding(ids, tv, yv, 2.0)
    L.assert_within(yv, *M.embedding(ids, table, 2.0), "y")
    assert int(ybuf.isnan().sum()) == ybuf.numel() - m * d
    for accumulate in (False, True):
        gv.zero_()
        edkm.embedding_backward(ids, dyv, gv, 2.0, accumulate)
        L.assert_within(gv, *M.embedding_grad(ids, dy, v, 2.0), "dtable")
        assert int(gbuf.isnan().sum()) == gbuf.numel() - v * d


def test_rows_of_no_token_may_hold_anything():
    """A token that stands for none takes nothing from dy, whatever is there."""
    ids = torch.tensor([3, -100, 3, 9, 4], device=DEV)
    dy = randn(1, 5, 40, dtype=torch.float16)
    ref, tol = M.embedding_grad(ids, dy, 9, 1.0)
    dy[1] = float("nan")
    dy[3] = float("inf")
    g = torch.empty(9, 40, dtype=torch.float16, device=DEV)
    edkm.embedding_backward(ids, dy, g)
    L.assert_within(g, ref, tol, "dtable")


@pytest.mark.parametrize("bits", [1, 2, 3, 4])
@pytest.mark.parametrize("fmt,m,v,d", [("fp16", 1, 50, 64), ("bf16", 33, 41, 77), ("fp16", 700, 129, 1001)])
def test_palette_embedding(bits, fmt, m, v, d):
    say("palette embedding", bits, fmt, m, v, d)
    dt = L.DT[fmt]
    idx, packed, lut = L.palette(v, d, bits, 3)
    ids = tokens(1, m, v)
    lut16 = torch.from_numpy(lut).to(DEV).to(dt)
    table = lut16[torch.from_numpy(idx).to(DEV).long()].view(v, d)
    for scale in (1.0, 3.3):
        y = torch.empty(m, d, dtype=dt, device=DEV)
        edkm.palette_embedding(ids, torch.from_numpy(packed).to(DEV), torch.from_numpy(lut).to(DEV), v, y, scale)
        L.assert_within(y, *M.embedding(ids, table, scale), "y")
        f = function.palette_embedding(ids.view(1, m), torch.from_numpy(packed).to(DEV), torch.from_numpy(lut).to(DEV), v, d, scale, dt)
        assert torch.equal(f, y.view(1, m, d))


def test_embedding_past_32_bits():
    """Offsets of a table and of outputs past 2^32 bytes."""
    v, d, m = 70001, 32768, 5
    say("embedding past 32 bits")
    table = torch.empty(v, d, dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([0, v - 1, 65537, v - 1, v], device=DEV)
    for t in (0, 65537, v - 1):
        table[t] = randn(t, d, dtype=torch.bfloat16)
    y = torch.empty(m, d, dtype=torch.bfloat16, device=DEV)
    edkm.embedding(ids, table, y)
    assert torch.equal(y[:4], table[ids[:4]]) and not bool(y[4].any())
    dy = randn(9, m, d, dtype=torch.bfloat16)
    table.fill_(float("nan"))
    edkm.embedding_backward(ids, dy, table)
    assert torch.equal(table[0], dy[0]) and torch.equal(table[65537], dy[2])
    assert torch.equal(table[v - 1], (dy[1].float() + dy[3].float()).bfloat16())
    assert float(table.view(-1)[:: 4099].float().abs().sum().isnan()) == 0.0


def test_embedding_of_no_tokens():
    say("embedding of nothing")
    dt = torch.bfloat16
    ids, table = torch.empty(0, dtype=torch.int64, device=DEV), randn(1, 70, 40, dtype=dt).requires_grad_()
    y = function.embedding(ids, table)
    assert y.shape == (0, 40)
    g, = torch.autograd.grad(y, table, torch.empty_like(y))
    assert not bool(g.any())
    old = randn(2, 70, 40, dtype=dt)
    more = old.clone()
    edkm.embedding_backward(ids, torch.empty(0, 40, dtype=dt, device=DEV), more, accumulate=True)
    assert torch.equal(old, more)
    assert function.embedding(torch.empty(2, 0, 3, dtype=torch.int32, device=DEV), table).shape == (2, 0, 3, 40)


# ---------------------------------------------------------------------------
# norms

NORM = [(1, 1), (1, 4096), (3, 7), (5, 64), (2, 511), (130, 512), (70, 513), (9, 1024), (33, 1025), (300, 1333), (40, 2049), (17, 4097),
        (6, 8192), (5, 8193), (3, 16384), (700, 256), (2500, 72),
        # more rows than a backward's workgroups
        (9000, 100), (8200, 65), (5000, 200), (4200, 500), (2100, 600), (1100, 1101), (600, 2104), (300, 4203), (270, 8200)]


@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
@pytest.mark.parametrize("m,n", NORM)
def test_residual_norm(fmt, m, n):
    dt, eps = L.DT[fmt], 1e-5
    for case, (block, post, gate) in enumerate([(False, False, None), (True, False, None), (True, True, "vector"), (True, False, "matrix"),
                                                (True, True, "matrix")]):
        say("norm", fmt, m, n, block, post, gate)
        r, w = randn(1, m, n, dtype=dt, scale=2.0), 1 + randn(2, n, dtype=dt, scale=0.3)
        u = randn(3, m, n, dtype=dt) if block else None
        p = 1 + randn(4, n, dtype=dt, scale=0.3) if post else None
        g = None if gate is None else randn(5, *((n,) if gate == "vector" else (m, n)), dtype=dt)
        dy, dh = (randn(6, m, n, dtype=dt) if case != 1 else None), (randn(7, m, n, dtype=dt) if case != 0 else None)
        y, h = torch.empty_like(r), torch.empty_like(r) if block else None
        edkm.residual_norm(r, w, y, h, u, p, g, 0.75, eps)
        rh, ry, th, ty = M.residual_norm(r, u, w, p, g, 0.75, eps)
        L.assert_within(y, ry, ty, "y")
        if block:
            L.assert_within(h, rh, th, "h")
        out = dict(dresidual=torch.empty_like(r), dweight=torch.empty_like(w))
        if block:
            out["dblock"] = torch.empty_like(u)
        if post:
            out["dpost_weight"] = torch.empty_like(p)
        if gate:
            out["dgate"] = torch.empty_like(g)
        edkm.residual_norm_backward(dy, dh, r, w, u, p, g, 0.75, eps, **out)
        names = {"dresidual": "dr", "dweight": "dw", "dblock": "du", "dpost_weight": "dpost", "dgate": "dgate"}
        for key, (ref, tol) in M.residual_norm_grads(dy, dh, r, u, w, p, g, 0.75, eps).items():
            mine = [o for o in out if names[o] == key]
            if mine:
                L.assert_within(out[mine[0]], ref, tol, key)
        again = {k: torch.empty_like(v) for k, v in out.items()}
        edkm.residual_norm_backward(dy, dh, r, w, u, p, g, 0.75, eps, **again)
        assert all(torch.equal(out[k], again[k]) for k in out)


@pytest.mark.parametrize("n,lead,gap", [(100, 1, 3), (1333, 8, 3), (4096, 8, 8), (70, 3, 0)])
def test_norm_views_in_nan_buffers(n, lead, gap):
    dt, m, eps = torch.float16, 19, 1e-6
    say("norm views", n, lead, gap)
    r, u, g, dy, dh = (randn(i, m, n, dtype=dt) for i in range(5))
    w, p = 1 + randn(6, n, dtype=dt, scale=0.2), 1 + randn(7, n, dtype=dt, scale=0.2)
    rv, uv, gv, dyv, dhv = (inside(t, lead, gap)[1] for t in (r, u, g, dy, dh))
    bufs = [inside(torch.zeros_like(r), lead, gap) for _ in range(4)]
    (hb, hv), (yb, yv), (drb, drv), (dub, duv) = bufs
    edkm.residual_norm(rv, w, yv, hv, uv, p, gv, 0.5, eps)
    rh, ry, th, ty = M.residual_norm(r, u, w, p, g, 0.5, eps)
    L.assert_within(hv, rh, th, "h")
    L.assert_within(yv, ry, ty, "y")
    edkm.residual_norm_backward(dyv, dhv, rv, w, uv, p, gv, 0.5, eps, drv, duv)
    ref = M.residual_norm_grads(dy, dh, r, u, w, p, g, 0.5, eps)
    L.assert_within(drv, *ref["dr"], "dr")
    L.assert_within(duv, *ref["du"], "du")
    for b, _ in bufs:
        assert int(b.isnan().sum()) == b.numel() - m * n


def test_norm_in_place_and_without_rows():
    say("norm in place")
    dt, m, n = torch.bfloat16, 40, 600
    r, u, w, p = randn(1, m, n, dtype=dt), randn(2, m, n, dtype=dt), randn(3, n, dtype=dt), randn(4, n, dtype=dt)
    h, y = torch.empty_like(r), torch.empty_like(r)
    edkm.residual_norm(r, w, y, h, u, p, None, 0.5)
    for own in (0, 1):
        r2, u2, y2 = r.clone(), u.clone(), torch.empty_like(y)
        edkm.residual_norm(r2, w, y2, u2 if own else r2, u2, p, None, 0.5)
        assert torch.equal(u2 if own else r2, h) and torch.equal(y2, y)
    dy, dh = randn(5, m, n, dtype=dt), randn(6, m, n, dtype=dt)
    dr, du = torch.empty_like(r), torch.empty_like(r)
    edkm.residual_norm_backward(dy, dh, r, w, u, p, None, 0.5, dresidual=dr, dblock=du)
    a, b, u2 = dy.clone(), dh.clone(), u.clone()
    edkm.residual_norm_backward(a, dh, r, w, u2, p, None, 0.5, dresidual=a, dblock=u2)
    assert torch.equal(a, dr) and torch.equal(u2, du)
    edkm.residual_norm_backward(dy, b, r, w, u, p, None, 0.5, dresidual=b)
    assert torch.equal(b, dr)
    r2 = r.clone()
    edkm.residual_norm_backward(dy, dh, r2, w, u, p, None, 0.5, dresidual=r2)
    assert torch.equal(r2, dr)
    none = torch.empty(0, n, dtype=dt, device=DEV)
    dw, dp, dg = (torch.ones(n, dtype=dt, device=DEV) for _ in range(3))
    edkm.residual_norm(none, w, none, none, none, p, w)
    edkm.residual_norm_backward(none, none, none, w, none, p, w, dweight=dw, dpost_weight=dp, dgate=dg)
    assert not bool(dw.any()) and not bool(dp.any()) and not bool(dg.any())


def test_norm_of_zeros_and_a_row_of_nan():
    dt, n = torch.float16, 300
    r = randn(1, 4, n, dtype=dt)
    r[1] = 0
    r[2, 5] = float("nan")
    w = torch.ones(n, dtype=dt, device=DEV)
    y = torch.empty_like(r)
    edkm.residual_norm(r, w, y)
    assert not bool(y[1].any()) and bool(y[2].isnan().all()) and bool(y[0].isfinite().all()) and bool(y[3].isfinite().all())


# ---------------------------------------------------------------------------
# cross entropy

LOSS = [(1, 1, 1), (1, 300, 64), (2, 17, 33), (7, 1003, 1337), (65, 64, 200), (64, 65, 8), (129, 2000, 96), (300, 513, 72), (257, 1030, 520),
        (1001, 1003, 777), (20, 9000, 1500)]


@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
@pytest.mark.parametrize("m,n,k", LOSS)
def test_cross_entropy(fmt, m, n, k, reduction):
    dt = L.DT[fmt]
    say("loss", fmt, m, n, k, reduction)
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=2 * k ** -0.5)
    targets = tokens(3, m, n, "log" if m > 1 else "one", torch.int32 if n % 2 else torch.int64)
    loss, lse = torch.empty(m if reduction == "none" else 1, device=DEV), torch.full((m,), float("nan"), device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse, reduction)
    ref, tol, rl, tl = M.cross_entropy(x, w, targets, reduction)
    L.assert_within(loss, ref.view(-1), tol.view(-1), "loss")
    L.assert_within(lse, rl, tl, "lse")
    dloss = torch.rand(m, device=DEV) - 0.3 if reduction == "none" else torch.tensor([0.7], device=DEV)
    if reduction == "none" and m > 4:
        dloss[4] = 0
    dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, dx, dw, reduction)
    for key, (ref, tol) in M.cross_entropy_grads(dloss, x, w, targets, reduction).items():
        L.assert_within({"dx": dx, "dw": dw}[key], ref, tol, key)
    dx2, dw2 = torch.empty_like(x), torch.empty_like(w)
    edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, dx2, None, reduction)
    edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, None, dw2, reduction)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
@pytest.mark.parametrize("m,n,k", [(16, 500, 300), (17, 500, 300), (1024, 300, 72), (1025, 300, 72), (40, 1000, 4096), (1300, 2100, 264),
                                   (2048, 4100, 512), (1100, 16640, 1032), (2000, 16384, 2048), (4096, 1000, 128), (64, 40000, 96), (8192, 200, 40), (8193, 200, 40)])
def test_cross_entropy_by_every_plan(fmt, m, n, k):
    """Sizes on both sides of each choice: few tokens and the list's length, tiles of 64, 128 and
    256, with the depths of one of the products split and not."""
    dt = L.DT[fmt]
    say("loss plans", fmt, m, n, k)
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=2 * k ** -0.5)
    targets = tokens(3, m, n)
    loss, lse = torch.empty(1, device=DEV), torch.full((m,), float("nan"), device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse, "mean")
    ref, tol, rl, tl = M.cross_entropy(x, w, targets, "mean")
    L.assert_within(loss, ref.view(1), tol.view(1), "loss")
    L.assert_within(lse, rl, tl, "lse")
    each = torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, each)
    ref, tol, _, _ = M.cross_entropy(x, w, targets, "none")
    L.assert_within(each, ref, tol, "losses")
    dloss, dx, dw = torch.full((1,), 512.0, device=DEV), torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, dx, dw, "mean")
    for key, (ref, tol) in M.cross_entropy_grads(dloss, x, w, targets, "mean").items():
        L.assert_within({"dx": dx, "dw": dw}[key], ref, tol, key)


@pytest.mark.parametrize("m,n,k,lead,gap", [(70, 200, 96, 1, 3), (70, 200, 96, 8, 8), (70, 201, 97, 3, 0), (300, 520, 136, 8, 4),
                                            (40, 1000, 4096, 1, 3), (9, 300, 264, 1, 3)])
def test_cross_entropy_views_in_nan_buffers(m, n, k, lead, gap):
    dt = torch.bfloat16
    say("loss views", m, n, k, lead, gap)
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=0.1)
    targets = tokens(3, m, n)
    _, xv = inside(x, lead, gap)
    _, wv = inside(w, lead, gap)
    xbuf, dxv = inside(torch.zeros_like(x), lead, gap)
    loss, lse = torch.empty(1, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(xv, wv, targets, loss, lse, "mean")
    ref, tol, _, _ = M.cross_entropy(x, w, targets, "mean")
    L.assert_within(loss, ref.view(1), tol.view(1), "loss")
    dwbuf = torch.full((lead + n * k + 16,), float("nan"), dtype=dt, device=DEV)
    dw = dwbuf[lead:lead + n * k].view(n, k)
    dloss = torch.ones(1, device=DEV)
    edkm.linear_cross_entropy_backward(dloss, xv, wv, targets, lse, dxv, dw, "mean")
    ref = M.cross_entropy_grads(dloss, x, w, targets, "mean")
    L.assert_within(dxv, *ref["dx"], "dx")
    L.assert_within(dw, *ref["dw"], "dw")
    assert int(xbuf.isnan().sum()) == xbuf.numel() - m * k
    assert int(dwbuf.isnan().sum()) == dwbuf.numel() - n * k


@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
def test_rows_without_a_target_may_hold_anything(reduction):
    """NaN and Inf in rows that do not count (no target, or no gradient) reach nothing."""
    dt, m, n, k = torch.bfloat16, 50, 300, 136
    say("masked nan", reduction)
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=0.1)
    targets = tokens(3, m, n)
    targets[7], targets[8] = -100, n
    clean = x.clone()
    x[7], x[8] = float("nan"), float("inf")
    loss, lse = torch.empty(m if reduction == "none" else 1, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse, reduction)
    ref, tol, _, _ = M.cross_entropy(clean, w, targets, reduction)
    L.assert_within(loss, ref.view(-1), tol.view(-1), "loss")
    dloss = torch.rand(m, device=DEV) + 0.1 if reduction == "none" else torch.ones(1, device=DEV)
    if reduction == "none":
        targets[9], dloss[9] = 5, 0.0
        x[9] = float("nan")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, dx, dw, reduction)
    ref = M.cross_entropy_grads(dloss, clean, w, targets, reduction)
    L.assert_within(dx, *ref["dx"], "dx")
    L.assert_within(dw, *ref["dw"], "dw")


def test_no_targets_and_no_tokens():
    dt, n, k = torch.float16, 90, 72
    w = randn(1, n, k, dtype=dt)
    for m in (0, 5):
        say("no targets", m)
        x = torch.full((m, k), float("nan"), dtype=dt, device=DEV)
        targets = torch.full((m,), -100, device=DEV)
        for reduction in ("none", "sum", "mean"):
            loss, lse = torch.ones(m if reduction == "none" else 1, device=DEV), torch.ones(m, device=DEV)
            edkm.linear_cross_entropy(x, w, targets, loss, lse, reduction)
            assert not bool(loss.any()) and not bool(lse.any())
            dx, dw = torch.ones_like(x), torch.ones_like(w)
            edkm.linear_cross_entropy_backward(torch.ones_like(loss), x, w, targets, lse, dx, dw, reduction)
            assert not bool(dx.any()) and not bool(dw.any())


def test_a_row_of_nan_stays_in_its_row_of_dx():
    dt, m, n, k = torch.float16, 40, 200, 64
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=0.2)
    targets = tokens(3, m, n, "one")
    x[3, 2] = float("nan")
    loss, lse, dx = torch.empty(m, device=DEV), torch.empty(m, device=DEV), torch.empty_like(x)
    edkm.linear_cross_entropy(x, w, targets, loss, lse)
    edkm.linear_cross_entropy_backward(torch.ones(m, device=DEV), x, w, targets, lse, dx)
    keep = [i for i in range(m) if i != 3]
    assert bool(loss[3].isnan()) and bool(dx[3].isnan().all()) and bool(loss[keep].isfinite().all()) and bool(dx[keep].isfinite().all())


def test_large_and_infinite_logits():
    """Logits of thousands: the loss keeps its digits; a logit of -Inf has no share."""
    dt, k = torch.bfloat16, 64
    x = torch.zeros(2, k, dtype=dt, device=DEV)
    x[:, 0], x[1, 1] = 100.0, 1.0
    w = torch.zeros(70, k, dtype=dt, device=DEV)
    w[3, 0], w[5, 0], w[69, 0] = 90.0, -90.0, 90.0
    targets = torch.tensor([3, 5], device=DEV)
    loss, lse = torch.empty(2, device=DEV), torch.empty(2, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse)
    ref, tol, _, _ = M.cross_entropy(x, w, targets, "none")
    L.assert_within(loss, ref, tol, "loss")
    w[7, 1] = -float("inf")
    x[0, 1] = 1.0
    edkm.linear_cross_entropy(x, w, targets, loss, lse)
    L.assert_within(loss, ref, tol, "loss with -Inf")


def test_pieces_of_the_vocabulary_and_of_the_tokens():
    """Sizes of which the gradient takes several pieces and the forward several launches."""
    dt, m, n, k = torch.bfloat16, 33000, 9001, 40
    say("pieces", m, n, k)
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=0.3)
    targets = tokens(3, m, n)
    loss, lse = torch.empty(1, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse, "mean")
    dloss, dx, dw = torch.ones(1, device=DEV), torch.empty_like(x), torch.empty_like(w)
    edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, dx, dw, "mean")
    there = (targets >= 0) & (targets < n)
    count, total, gw, ew = int(there.sum()), 0.0, 0.0, 0.0
    for a in range(0, m, 3000):
        s = slice(a, a + 3000)
        ref, _, _, _ = M.cross_entropy(x[s], w, targets[s], "sum")
        total += ref
        g = M.cross_entropy_grads(torch.full((1,), 1.0 / count, device=DEV), x[s], w, targets[s], "sum")
        L.assert_within(dx[s], *g["dx"], "dx")
        gw, ew = gw + g["dw"][0], ew + g["dw"][1]      # the bounds of a sum are at most the bounds' sum
    assert abs(float(loss) - float(total / count)) <= 1e-5 * float(total / count)
    L.assert_within(dw, gw, ew + gw.abs() * L.half(dt), "dw")


@pytest.mark.parametrize("m", [3, 40])
def test_cross_entropy_past_32_bits(m):
    """A vocabulary's weights and their gradient of more than 2^32 bytes; words at both ends."""
    dt, n, k = torch.bfloat16, 70001, 32768
    say("loss past 32 bits", m)
    x = randn(1, m, k, dtype=dt)
    w = torch.empty(n, k, dtype=dt, device=DEV)
    for a in range(0, n, 10000):
        w[a:a + 10000] = randn(a + 7, min(10000, n - a), k, dtype=dt, scale=0.01)
    targets = torch.randint(0, n, (m,), device=DEV)
    targets[:3] = torch.tensor([n - 1, 0, 66000])
    z = torch.cat([x.double() @ w[a:a + 4000].double().t() for a in range(0, n, 4000)], 1)
    want = torch.logsumexp(z, 1) - z.gather(1, targets[:, None])[:, 0]
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse)
    # a logit is off by less than (k + 2) 2^-23 times its terms' magnitudes, about k 0.8 0.008
    assert float((loss.double() - want).abs().max()) <= 2 * (k + 2) * 2.0 ** -23 * k * 0.0064
    dw, dx = torch.empty_like(w), torch.empty_like(x)
    edkm.linear_cross_entropy_backward(torch.ones(m, device=DEV), x, w, targets, lse, dx, dw)
    dz = torch.softmax(z, 1)
    dz[torch.arange(m, device=DEV), targets] -= 1
    rows = torch.tensor([0, 1, 32767, 65535, 65536, 66000, n - 2, n - 1], device=DEV)
    ref, mag = dz[:, rows].t() @ x.double(), dz[:, rows].abs().t() @ x.double().abs()
    # dz's rounding and its own fp32 error (its logit's, relative), and the sum's and its rounding
    bound = mag * (L.half(dt) * 2 + 2 * (k + 2) * 2.0 ** -23 * k * 0.0064) + ref.abs() * L.half(dt) + 1e-30
    L.assert_within(dw[rows], ref, bound, "dw")
    assert bool(dx.isfinite().all()) and bool(dw[::997].isfinite().all())


# ---------------------------------------------------------------------------
# through autograd


@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
def test_a_run_of_all_three(fmt):
    """Tokens to a loss as a model runs them, with a table that is both ends; gradients of
    every leaf against 64-bit autograd."""
    dt, b, t, v, d = L.DT[fmt], 3, 37, 210, 72
    say("run of all three", fmt)
    ids = tokens(1, b * t, v).view(b, t)
    table = randn(2, v, d, dtype=dt, scale=0.3).requires_grad_()
    w0, w1, post = ((1 + randn(i, d, dtype=dt, scale=0.2)).requires_grad_() for i in (3, 4, 5))
    gate = randn(6, d, dtype=dt).requires_grad_()
    proj = randn(7, d, d, dtype=dt, scale=d ** -0.5).requires_grad_()
    targets = torch.where(torch.rand(b, t, device=DEV) < 0.2, -100, ids.roll(-1, 1))
    leaves, scale = [table, w0, w1, post, gate, proj], 256.0

    def exact(targets):
        q = [x.detach().double().requires_grad_() for x in leaves]
        tb, a0, a1, ps, gt, pj = q
        ok = (ids >= 0) & (ids < v)
        r = torch.where(ok[..., None], tb[ids.clamp(0, v - 1)], 0.0) * 2
        u = torch.nn.functional.silu(M.norm(r, a0, 1e-6).reshape(-1, d) @ pj.t()).view(b, t, d)
        h = r + 0.5 * gt * M.norm(u, ps, 1e-6)
        z = (M.norm(h, a1, 1e-6).reshape(-1, d) @ tb.t())
        count = (targets >= 0) & (targets < v)
        loss = torch.nn.functional.cross_entropy(z, torch.where(count, targets, -100).view(-1)) + h.pow(2).mean() * 0.01
        return loss.detach(), torch.autograd.grad(loss * scale, [*q, u])
    if fmt == "fp16":
        # A row of zeros passes its gradient on 1 / sqrt(eps) = 1000 times as large in each norm: past
        # fp16's largest number at the block's output, if a token that stands for none has a target.
        assert float(exact(targets)[1][-1].abs().max()) > 65504
        targets = torch.where((ids >= 0) & (ids < v), targets, -100)
    r = function.embedding(ids, table, 2.0)
    y = function.linear(function.rms_norm(r, w0), proj, activation="silu")
    h, y = function.residual_norm(r, y, w1, post, gate, 0.5)
    loss = function.linear_cross_entropy(y, table, targets) + (h.float().pow(2).mean() * 0.01)
    assert r.shape == (b, t, d) and h.shape == r.shape and loss.dtype == torch.float32
    mine = torch.autograd.grad(loss * scale, leaves)
    loss = loss.detach()
    ref, grads = exact(targets)
    # the chain rounds to 16 bits some ten times on its way: a root of tens of half steps, relative to the whole
    assert abs(float(loss) - float(ref)) <= 8 * L.half(dt) * abs(float(ref))
    for name, a, e in zip(("table", "w0", "w1", "post", "gate", "proj"), mine, grads):
        off = float((a.double() - e).norm() / e.norm())
        assert off <= 8 * L.half(dt), (name, off)


def test_gradients_against_differences():
    """The analytic gradients against central differences of the operators' own 64-bit
    forms along random directions (the forms are what the kernels are held to above)."""
    dt, m, n, k = torch.float16, 6, 50, 24
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=0.3)
    targets = tokens(3, m, n, "flat")
    targets[0] = 4
    g = M.cross_entropy_grads(torch.ones(1, device=DEV), x, w, targets, "mean")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    loss, lse = torch.empty(1, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse, "mean")
    edkm.linear_cross_entropy_backward(torch.ones(1, device=DEV), x, w, targets, lse, dx, dw, "mean")
    for mine, ref, at in ((dx, g["dx"], 0), (dw, g["dw"], 1)):
        v = randn(9, *ref[0].shape, dtype=torch.float64)
        e = 1e-5
        f = [M.cross_entropy(*(t.double() + (s * e * v if i == at else 0) for i, t in enumerate((x, w))), targets, "mean")[0] for s in (1, -1)]
        slope = float((f[0] - f[1]) / (2 * e))
        assert abs(float((ref[0] * v).sum()) - slope) <= 1e-7 * float((ref[0] * v).abs().sum())
        assert abs(float((mine.double() * v).sum()) - slope) <= float((ref[1] * v.abs()).sum()) + 1e-7 * float((ref[0] * v).abs().sum())
    r, u, p, q, gt = (randn(i, 5, 30, dtype=torch.float64) for i in range(5))
    w1, post = 1 + randn(7, 30, dtype=torch.float64, scale=0.2), 1 + randn(8, 30, dtype=torch.float64, scale=0.2)

    def f(args):
        h, y, _, _ = M.residual_norm(*args, 0.5, 1e-5)
        return (h * p).sum() + (y * q).sum()
    args = [r, u, w1, post, gt]
    ref = M.residual_norm_grads(q, p, r, u, w1, post, gt, 0.5, 1e-5)
    for i, key in enumerate(("dr", "du", "dw", "dpost", "dgate")):
        v = randn(20 + i, *args[i].shape, dtype=torch.float64)
        e = 1e-5
        ends = [f([t + (s * e * v if j == i else 0) for j, t in enumerate(args)]) for s in (1, -1)]
        want, have = float((ends[0] - ends[1]) / (2 * e)), float((ref[key][0] * v).sum())
        assert abs(want - have) <= 1e-7 * float((ref[key][0] * v).abs().sum()), key


def test_autograd_forms():
    """Broadcast and strided gradients, leaves that need none, and what is refused."""
    dt = torch.bfloat16
    say("autograd forms")
    ids = tokens(1, 24, 50).view(4, 6)
    table = randn(2, 50, 40, dtype=dt).requires_grad_()
    y = function.embedding(ids, table)
    g, = torch.autograd.grad(y.float().sum(), table)
    ref, tol = M.embedding_grad(ids.view(-1), torch.ones(24, 40, dtype=dt, device=DEV), 50, 1.0)
    L.assert_within(g, ref, tol, "broadcast dy")
    dy = randn(3, 6, 4, 40, dtype=dt).transpose(0, 1)
    g, = torch.autograd.grad(function.embedding(ids, table), table, dy)
    L.assert_within(g, *M.embedding_grad(ids.view(-1), dy.reshape(24, 40), 50, 1.0), "strided dy")
    x, w = randn(4, 4, 6, 40, dtype=dt).requires_grad_(), randn(5, 50, 40, dtype=dt, scale=0.2)
    loss = function.linear_cross_entropy(x, w, ids, "none")
    assert loss.shape == ids.shape
    gx, = torch.autograd.grad(loss.sum(), x)
    ref = M.cross_entropy_grads(torch.ones(24, device=DEV), x.detach().view(24, 40), w, ids.view(-1), "none")
    L.assert_within(gx.view(24, 40), *ref["dx"], "dx")
    r, u = randn(6, 4, 6, 40, dtype=dt).requires_grad_(), randn(7, 4, 6, 40, dtype=dt)
    weight = torch.ones(40, dtype=dt, device=DEV, requires_grad=True)
    gate = randn(8, 4, 6, 40, dtype=dt).requires_grad_()
    h, y = function.residual_norm(r, u, weight, None, gate)
    for out in (h, y):         # one of the two outputs used, a block without gradient
        gs = torch.autograd.grad(out.float().sum(), [r, gate], retain_graph=True)
        one = torch.ones(24, 40, dtype=dt, device=DEV)
        ref = M.residual_norm_grads(one if out is y else None, one if out is h else None, r.detach().view(24, 40), u.view(24, 40), weight.detach(),
                                    None, gate.detach().view(24, 40), 1.0, 1e-6)
        L.assert_within(gs[0].view(24, 40), *ref["dr"], "dr")
        L.assert_within(gs[1].view(24, 40), *ref["dgate"], "dgate")
    again = torch.autograd.grad(function.rms_norm(r, weight).float().sum(), r, create_graph=True)[0]
    with pytest.raises(RuntimeError, match="differentiated again"):
        again.float().sum().backward()
    bad = function.rms_norm(r, weight)
    with torch.no_grad():
        r.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        bad.float().sum().backward()


def test_another_stream_and_a_captured_step():
    """On another stream with an own workspace, and captured: every replay on new inputs
    gives what the eager calls give."""
    dt, m, v, d = torch.float16, 300, 400, 136
    say("streams and graphs")
    ids, table = tokens(1, m, v), randn(2, v, d, dtype=dt)
    w, u = 1 + randn(3, d, dtype=dt, scale=0.1), randn(4, m, d, dtype=dt)
    dloss = torch.ones(1, device=DEV)
    ws = [torch.empty(max(256, n), dtype=torch.uint8, device=DEV) for n in (
        edkm.linear_cross_entropy_workspace_bytes(m, v, d), edkm.linear_cross_entropy_backward_workspace_bytes(m, v, d),
        edkm.residual_norm_backward_workspace_bytes(m, d), edkm.embedding_backward_workspace_bytes(m, v, d))]

    def buffers():
        e = lambda *s, t=dt: torch.empty(s, dtype=t, device=DEV)  # noqa: E731
        return dict(r=e(m, d), h=e(m, d), y=e(m, d), loss=e(1, t=torch.float32), lse=e(m, t=torch.float32), dy=e(m, d), dtab=e(v, d), dr=e(m, d),
                    du=e(m, d), dw=e(d), dt2=e(v, d))

    def step(o, s=None):
        edkm.embedding(ids, table, o["r"], 1.5, stream=s)
        edkm.residual_norm(o["r"], w, o["y"], o["h"], u, None, None, 0.5, stream=s)
        edkm.linear_cross_entropy(o["y"], table, ids, o["loss"], o["lse"], "mean", ws[0], s)
        edkm.linear_cross_entropy_backward(dloss, o["y"], table, ids, o["lse"], o["dy"], o["dtab"], "mean", ws[1], s)
        edkm.residual_norm_backward(o["dy"], None, o["r"], w, u, None, None, 0.5, dresidual=o["dr"], dblock=o["du"], dweight=o["dw"],
                                    workspace=ws[2], stream=s)
        edkm.embedding_backward(ids, o["dr"], o["dt2"], 1.5, workspace=ws[3], stream=s)

    side = torch.cuda.Stream()
    base, o = buffers(), buffers()
    step(base)
    side.wait_stream(torch.cuda.current_stream())
    step(o, side)
    torch.cuda.synchronize()
    assert all(torch.equal(base[k], o[k]) for k in o)
    with pytest.raises(ValueError, match="workspace"):
        edkm.embedding_backward(ids, o["dr"], o["dt2"], stream=side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(o)
    for i in range(4):
        with torch.no_grad():
            ids.copy_(tokens(10 + i, m, v))
            table.copy_(randn(20 + i, v, d, dtype=dt))
        for t in o.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        step(base)
        torch.cuda.synchronize()
        for k in o:
            assert torch.equal(base[k], o[k]), (i, k)


def test_a_captured_step_through_autograd():
    dt, m, v, d = torch.bfloat16, 70, 90, 64
    say("captured autograd")
    ids = tokens(1, m, v)
    table, w = randn(2, v, d, dtype=dt).requires_grad_(), torch.ones(d, dtype=dt, device=DEV, requires_grad=True)

    def step():
        loss = function.linear_cross_entropy(function.rms_norm(function.embedding(ids, table), w), table, ids)
        return (loss, *torch.autograd.grad(loss, [table, w]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        ids.copy_(tokens(5 + i, m, v))
        with torch.no_grad():
            table.copy_(randn(30 + i, v, d, dtype=dt))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)


def test_cross_entropy_of_the_largest_vocabulary():
    """Words up to the largest number a size can be, of rows that have to be copied: numbers of rows
    that a step of 8192 takes past 2^31."""
    dt, n = torch.bfloat16, 2 ** 31 - 1 - 1024
    say("largest vocabulary")
    x, w = torch.ones(1, 1, dtype=dt, device=DEV), torch.zeros(n, 1, dtype=dt, device=DEV)
    w[5], w[n - 1] = 1.0, 2.0
    targets = torch.tensor([n - 1], device=DEV)
    total = n - 2 + np.exp(1.0) + np.exp(2.0)
    loss, lse = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse)
    # up to 2^17 + 30 additions of equal numbers one after another, exact while the sum is below 2^24
    # of them; what is left is the logarithm's and lse's own rounding, and a few ulps of the sum
    assert abs(float(lse) - np.log(total)) <= 4 * M.U * np.log(total) + 40 * M.U
    assert abs(float(loss) - (np.log(total) - 2)) <= 4 * M.U * np.log(total) + 40 * M.U
    torch.cuda.empty_cache()
    dx, dw = torch.empty_like(x), torch.full_like(w, float("nan"))
    edkm.linear_cross_entropy_backward(torch.ones(1, device=DEV), x, w, targets, lse, dx, dw)
    # lse's error is p's, relative; dz and dw are rounded once each
    near = 2 * L.half(dt) + 2 * M.U * np.log(total) + 40 * M.U
    for at, ref in ((5, np.exp(1.0) / total), (n - 1, np.exp(2.0) / total - 1), (0, 1 / total), (n - 2, 1 / total)):
        assert abs(float(dw[at]) - ref) <= near * abs(ref), at
    same = sum(int((dw[a:a + 2 ** 28] == dw[0]).sum()) for a in range(0, n, 2 ** 28))
    assert same == n - 2
    ref = np.exp(1.0) / total + 2 * (np.exp(2.0) / total - 1)
    assert abs(float(dx) - ref) <= near * abs(ref)
    del w, dw
    torch.cuda.empty_cache()


@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("m", [0, 5, 9000])
def test_no_targets_in_a_workspace_of_nan(m, reduction):
    """What a backward takes from its list of no tokens is written there, not found."""
    dt, n, k = torch.bfloat16, 90, 72
    say("no targets, workspace of NaN", m, reduction)
    nans = lambda size: torch.full((size,), 255, dtype=torch.uint8, device=DEV)  # noqa: E731
    x, w = torch.full((m, k), float("nan"), dtype=dt, device=DEV), randn(1, n, k, dtype=dt)
    targets = torch.full((m,), -100, device=DEV)
    loss, lse = torch.ones(m if reduction == "none" else 1, device=DEV), torch.ones(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse, reduction, nans(edkm.linear_cross_entropy_workspace_bytes(m, n, k)))
    assert not bool(loss.any()) and not bool(lse.any())
    dx, dw = torch.ones_like(x), torch.ones_like(w)
    edkm.linear_cross_entropy_backward(torch.ones_like(loss), x, w, targets, lse, dx, dw, reduction,
                                       nans(edkm.linear_cross_entropy_backward_workspace_bytes(m, n, k)))
    assert not bool(dx.any()) and not bool(dw.any())


@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
@pytest.mark.parametrize("m", [5, 17, 64, 300, 1100, 9000])
def test_certain_tokens_have_no_loss(fmt, m):
    """A certain target has a loss of 0 and no gradient however large its logit is, by every kernel; of
    two words as large as each other each has half.  A token's logits are one product that is not 0,
    v or -v for v of 40 to 3040, so they are exact, and e^(-2 v) is at most 1.8e-35."""
    dt, n, k = L.DT[fmt], 500, 64
    say("certain tokens", fmt, m)
    g = torch.Generator(device=DEV).manual_seed(m)
    v = (40 + 3000 * torch.rand(m, generator=g, device=DEV)).to(dt)
    i, j = torch.arange(m, device=DEV), torch.arange(k, device=DEV)
    c = i % k
    x, w = torch.zeros(m, k, dtype=dt, device=DEV), -torch.ones(n, k, dtype=dt, device=DEV)
    x[i, c], w[j, j] = v, 1.0
    w[k + j[32:], j[32:]] = 1.0         # the columns from 32 on have two such words
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, c, loss, lse)
    ref = torch.where(c < 32, 0.0, np.log(2.0)).double()
    # the sum is 1 or 2, exactly; its logarithm is off by at most two ulps
    assert bool((loss >= 0).all())
    L.assert_within(loss, ref, ref * 2 * M.U, "loss")
    L.assert_within(lse, v.double() + ref, (v.double() + ref) * M.U, "lse")
    dloss, dx, dw = torch.full((m,), 1.0 / m, device=DEV), torch.empty_like(x), torch.empty_like(w)
    edkm.linear_cross_entropy_backward(dloss, x, w, c, lse, dx, dw)
    # half's error: lse's rounding, an ulp or two of e^, the rounding to 16 bits
    each = 0.5 * (v.double() * M.U + 8 * M.U + L.half(dt)) / m
    # both words of a pair have the same row of w: their shares, -1/2 and 1/2, cancel but for their errors
    L.assert_within(dx, torch.zeros_like(dx).double(), torch.where(c < 32, 0.0, 2 * each * (1 + L.half(dt)))[:, None].expand(m, k) + 1e-30 + L.tiny(dt), "dx")
    ref, tol = torch.zeros(n, k, dtype=torch.float64, device=DEV), torch.zeros(n, k, dtype=torch.float64, device=DEV)
    two = c >= 32
    half = 0.5 * v.double()[two] / m
    for row, sign in ((c, -1), (c + k, 1)):
        ref.index_put_((row[two], c[two]), sign * half, accumulate=True)
        tol.index_put_((row[two], c[two]), each[two] * v.double()[two], accumulate=True)
    tol = tol + ref.abs() * (L.half(dt) + (m + 4) * M.U) + 1e-30 + L.tiny(dt)
    L.assert_within(dw, ref, tol, "dw")


@pytest.mark.parametrize("m", [40, 2000, 9000])
def test_an_infinite_gradient_stays_in_its_token(m):
    """dx_i = g_i (p - onehot) W: an Inf or NaN among dL/dloss spoils its own row of dx and no other."""
    dt, n, k = torch.float16, 100, 64
    say("infinite dloss", m)
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=0.3)
    targets = tokens(3, m, n)
    targets[5:8] = torch.tensor([1, 2, 3], device=DEV)
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse)
    dloss = torch.rand(m, device=DEV) + 0.1
    for odd in ((float("inf"), 0.5, 0.5), (-float("inf"), float("nan"), float("inf"))):
        dloss[5:8] = torch.tensor(odd, device=DEV)
        dx = torch.empty_like(x)
        edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, dx)
        finite = dloss.isfinite()
        ref, tol = M.cross_entropy_grads(torch.where(finite, dloss, 0.0), x, w, targets, "none")["dx"]
        L.assert_within(dx[finite], ref[finite], tol[finite], "dx")
        assert not bool(dx[~finite].isfinite().any())
    # none that is finite: the rows of no target are still zeros
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    edkm.linear_cross_entropy_backward(torch.full_like(dloss, float("inf")), x, w, targets, lse, dx, dw)
    there = (targets >= 0) & (targets < n)
    assert not bool(dx[there].isfinite().any()) and not bool(dx[~there].any()) and not bool(dw.isfinite().any())


@pytest.mark.parametrize("m", [30, 9000])
@pytest.mark.parametrize("g", [1.3 * 2.0 ** -132, 1.7 * 2.0 ** -122, 1.9 * 2.0 ** 110])
@pytest.mark.parametrize("reduction", ["sum", "mean"])
def test_gradients_of_tiny_and_huge_scale(m, g, reduction):
    """dL/dloss down to fp32's subnormal numbers and up to where dx leaves bf16's range: what the
    gradients are scaled by keeps its digits."""
    dt, n, k = torch.bfloat16, 100, 64
    say("scale of dloss", m, g, reduction)
    x, w = randn(1, m, k, dtype=dt, scale=2.0 ** -12), randn(2, n, k, dtype=dt, scale=2.0 ** 12)
    targets = tokens(3, m, n)
    loss, lse = torch.empty(1, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse, reduction)
    dloss, dx, dw = torch.full((1,), g, dtype=torch.float64).float().to(DEV), torch.empty_like(x), torch.empty_like(w)
    edkm.linear_cross_entropy_backward(dloss, x, w, targets, lse, dx, dw, reduction)
    for key, (ref, tol) in M.cross_entropy_grads(dloss, x, w, targets, reduction).items():
        L.assert_within({"dx": dx, "dw": dw}[key], ref, tol, key)


def test_embedding_of_more_tokens_times_rows_than_a_matrix_holds():
    """2^22 + 1 tokens of a table of 2^18 rows: neither the table nor y is large."""
    dt, m, v, d = torch.bfloat16, (1 << 22) + 1, 1 << 18, 8
    say("embedding, many tokens and rows")
    ids = torch.randint(-5, v + 5, (m,), device=DEV)
    table, dy = randn(1, v, d, dtype=dt), randn(2, m, d, dtype=dt)
    y, g = torch.empty(m, d, dtype=dt, device=DEV), torch.empty_like(table)
    edkm.embedding(ids, table, y)
    there = (ids >= 0) & (ids < v)
    assert torch.equal(y, torch.where(there[:, None], table[ids.clamp(0, v - 1)], 0.0))
    edkm.embedding_backward(ids, dy, g)
    L.assert_within(g, *M.embedding_grad(ids, dy, v, 1.0), "dtable")
    idx, packed, lut = L.palette(v, d, 3, 3)
    edkm.palette_embedding(ids, torch.from_numpy(packed).to(DEV), torch.from_numpy(lut).to(DEV), v, y)
    table = torch.from_numpy(lut).to(DEV).to(dt)[torch.from_numpy(idx).to(DEV).long()].view(v, d)
    assert torch.equal(y, torch.where(there[:, None], table[ids.clamp(0, v - 1)], 0.0))


def test_norm_gradients_of_no_rows_are_zeros_whatever_the_vectors_hold():
    dt, n = torch.bfloat16, 70
    none = torch.empty(0, n, dtype=dt, device=DEV)
    odd = torch.full((n,), float("inf"), dtype=dt, device=DEV)
    odd[3::7] = float("nan")
    dw, dp, dg = (torch.ones(n, dtype=dt, device=DEV) for _ in range(3))
    edkm.residual_norm_backward(none, none, none, odd, none, odd, odd, dweight=dw, dpost_weight=dp, dgate=dg)
    assert not bool(dw.any()) and not bool(dp.any()) and not bool(dg.any())


@pytest.mark.parametrize("m", [3, 40, 1100])
def test_cross_entropy_past_32_bits_with_exact_logits(m):
    """A vocabulary's weights and their gradient of more than 2^32 bytes, held to bounds that a
    missing or misplaced value does not meet: x is not 0 in three columns, where both hold multiples
    of 1/4 up to 1, so that a logit is exact in fp32 and a row of dw has three values."""
    dt, n, k = torch.bfloat16, 70001, 32768
    say("loss past 32 bits, exact logits", m)
    at = torch.tensor([0, 16385, k - 1], device=DEV)
    g = torch.Generator(device=DEV).manual_seed(m)
    quarters = lambda rows: (torch.randint(1, 5, (rows, 3), generator=g, device=DEV)  # noqa: E731
                             * (1 - 2 * torch.randint(0, 2, (rows, 3), generator=g, device=DEV)) / 4).to(dt)
    x, w = torch.zeros(m, k, dtype=dt, device=DEV), torch.empty(n, k, dtype=dt, device=DEV)
    for a in range(0, n, 10000):
        w[a:a + 10000] = randn(a + 7, min(10000, n - a), k, dtype=dt)
    x[:, at], w[:, at] = quarters(m), quarters(n)
    targets = torch.randint(0, n, (m,), generator=g, device=DEV)
    targets[:3] = torch.tensor([n - 1, 0, 66000])
    z = x[:, at].double() @ w[:, at].double().t()
    lse_ref = torch.logsumexp(z, 1)
    want = lse_ref - z.gather(1, targets[:, None])[:, 0]
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    edkm.linear_cross_entropy(x, w, targets, loss, lse)
    # a term passes up to 18 additions in its block, 35 blocks of a thread and 22 joins, each with two
    # products by e^ (an ulp each, and two of its argument); logits are multiples of 1/16
    tol = 500 * M.U + 4 * M.U * lse_ref
    assert float(tol.max()) < 1 / 64
    L.assert_within(lse, lse_ref, tol, "lse")
    L.assert_within(loss, want, tol, "loss")
    dw, dx = torch.full_like(w, float("nan")), torch.full_like(x, float("nan"))
    edkm.linear_cross_entropy_backward(torch.ones(m, device=DEV), x, w, targets, lse, dx, dw)
    dz = torch.softmax(z, 1)
    dz[torch.arange(m, device=DEV), targets] -= 1
    # lse's error and e^'s own relative, the target's 1 by an ulp, then the rounding to 16 bits
    ed = dz.abs() * L.half(dt) + (dz.abs() + 1e-9) * (tol + 40 * M.U)[:, None] * (1 + L.half(dt))
    ed[torch.arange(m, device=DEV), targets] += 2 * M.U
    ref, mag = dz.t().contiguous() @ x[:, at].double(), dz.abs().t().contiguous() @ x[:, at].double().abs()
    bound = ed.t().contiguous() @ x[:, at].double().abs() + (m + 4) * M.U * mag
    bound = bound + ref.abs() * L.half(dt) + L.tiny(dt)
    assert float((bound < ref.abs()).double().mean()) > 0.9       # zeros would be refused
    L.assert_within(dw[:, at], ref, bound, "dw")
    dw[:, at] = 0
    assert not any(bool(dw[a:a + 10000].any()) for a in range(0, n, 10000))
    cols = torch.cat([at, torch.arange(5, k, 499, device=DEV)])
    wc = torch.cat([w[a:a + 10000][:, cols] for a in range(0, n, 10000)]).double()
    ref, mag = dz @ wc, dz.abs() @ wc.abs()
    # sums of a tile's depths, its parts and the pieces, whatever their order: by n ulps at most
    bound = ed @ wc.abs() + (n + 4) * M.U * mag
    bound = bound + ref.abs() * L.half(dt) + L.tiny(dt)
    assert float((bound < ref.abs()).double().mean()) > 0.9
    L.assert_within(dx[:, cols], ref, bound, "dx")
    assert bool(dx.isfinite().all())


@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
@pytest.mark.parametrize("m,n,k", [(8, 500, 304), (9, 500, 304), (16, 500, 304), (8, 500, 301), (9, 500, 301), (16, 500, 301), (17, 500, 301)])
def test_cross_entropy_of_few_tokens(fmt, m, n, k):
    """Both sides of the few tokens that take no tiles, with rows of whole pieces and without."""
    dt = L.DT[fmt]
    say("few tokens", fmt, m, n, k)
    x, w = randn(1, m, k, dtype=dt), randn(2, n, k, dtype=dt, scale=2 * k ** -0.5)
    targets = tokens(3, m, n, "flat")
    for reduction in ("none", "sum", "mean"):
        loss, lse = torch.empty(m if reduction == "none" else 1, device=DEV), torch.full((m,), float("nan"), device=DEV)
        edkm.linear_cross_entropy(x, w, targets, loss, lse, reduction)
        ref, tol, rl, tl = M.cross_entropy(x, w, targets, reduction)
        L.assert_within(loss, ref.view(-1), tol.view(-1), "loss")
        L.assert_within(lse, rl, tl, "lse")


@pytest.mark.parametrize("m,n,k,lead,gap", [(8, 300, 264, 1, 3), (8, 300, 264, 8, 8), (3, 300, 256, 3, 5), (16, 300, 261, 1, 3), (16, 300, 264, 8, 4)])
def test_cross_entropy_views_of_few_tokens(m, n, k, lead, gap):
    """The same for tokens that share a workgroup's words, and for the first that do not."""
    test_cross_entropy_views_in_nan_buffers(m, n, k, lead, gap)
