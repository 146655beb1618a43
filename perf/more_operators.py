"""The operators at a model's two ends and between its blocks, as cases that a timing
program can list, draw, prepare and run.

A case is a dict of plain values:

* ``kind``: which operator one pass calls.
  - ``embed``: rows of a 16-bit table by token, times a scale, and the table's gradient for
    a given dL/dy, through torch's autograd;
  - ``embed_add``: the gradient alone, added to the table's gradient so far;
  - ``embed_palette``: rows of a table stored as a palette (packed b-bit indices and a
    table of 2^b values), the served lookup;
  - ``loss``: softmax cross entropy of x W^T against target tokens;
  - ``norm``: h = r + scale * gate * N(u; post) and y = N(h; w), the step from one block to
    the next, N(v; w) = v / sqrt(mean(v^2) + eps) * w.
* ``embed*``: ``m`` tokens, ``v`` rows of ``d`` values, ``fmt``, ``index`` type of the
  tokens, ``scale``, ``bits`` of a palette, ``share`` of tokens outside the table.
* ``loss``: ``m`` tokens, ``n`` words, ``k`` inputs, ``fmt``, ``train`` (with the gradients
  of x and W), ``reduction``, ``share`` of tokens that do not count.
* ``norm``: ``m`` tokens of ``n`` values, ``fmt``, ``train``, ``post`` (the norm of the
  block's output), ``gate`` (none, vector, matrix), ``scale``.

Definitions.  A token outside the table has a row of zeros and no gradient; a target
outside the vocabulary has no loss and no gradient, and does not count in a mean (the
mean over none is 0).  All sums and functions are exact ones, and each output is rounded
once, at the end; a palette's weight is its table entry rounded to the 16-bit type.
"""
import math

import torch

own = False      # True: the framework's operators; False: their plain form

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
INDEX = {"int32": torch.int32, "int64": torch.int64}
EPS = 1e-6
OUTSIDE = -100           # the token that stands for none
_MOST = 8192 * 32000 * 4096


def _embed(name, kind, m, v, d, **kw):
    c = dict(name=name, kind=kind, m=m, v=v, d=d, fmt="bf16", index="int64", scale=1.0, bits=0, share=0.0)
    c.update(kw)
    return c


def _loss(name, m, n, k, **kw):
    c = dict(name=name, kind="loss", m=m, n=n, k=k, fmt="bf16", index="int64", train=True, reduction="mean", share=0.0)
    c.update(kw)
    return c


def _norm(name, m, n, **kw):
    c = dict(name=name, kind="norm", m=m, n=n, fmt="bf16", train=True, post=False, gate="none", scale=1.0)
    c.update(kw)
    return c


def listed():
    return [
        # the next token of one sequence from a served 3-bit embedding
        _embed("embed_palette_1", "embed_palette", 1, 32000, 4096, fmt="fp16", bits=3),
        # the embedding's training step on four sequences of 2048 tokens, scaled by sqrt(d)
        _embed("embed_8192", "embed", 8192, 32000, 4096, scale=64.0, share=0.02),
        # a small odd table, fp16
        _embed("embed_odd_fp16", "embed", 1001, 1003, 777, fmt="fp16", scale=0.5, share=0.1),
        # another micro-batch added to the gradient of a narrower table
        _embed("embed_add_65536", "embed_add", 65536, 50000, 1024),
        # one token's loss: scoring as it is generated
        _loss("loss_1", 1, 32000, 4096, train=False, reduction="none"),
        # the losses of a 512-token text
        _loss("loss_512", 512, 32000, 4096, train=False, reduction="none"),
        # a small odd head with a weight for each token
        _loss("loss_odd_fp16", 1001, 1003, 777, fmt="fp16", reduction="none", share=0.1),
        # a training step over a large vocabulary and a narrow model
        _loss("loss_2048_wide", 2048, 131072, 2048, share=0.25),
        # the training step of four sequences of 2048 tokens: the largest
        _loss("loss_8192", 8192, 32000, 4096, share=0.02),
        # between two blocks for one token
        _norm("norm_1", 1, 4096, train=False, post=True, gate="vector", scale=0.5),
        # between two blocks in the training of four sequences of 2048 tokens
        _norm("norm_8192", 8192, 4096, post=True, gate="vector", scale=0.5),
        # odd sizes, a gate for each token
        _norm("norm_odd_fp16", 1001, 1333, fmt="fp16", gate="matrix", scale=0.25),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random() + 0.5)))


def _size(rng, lo, hi):
    """A size of the range: a multiple of 64, a multiple of 8, or any."""
    n, step = _log(rng, lo, hi), rng.choice([64, 64, 8, 1])
    return min(hi, max(1, n // step * step)) if n >= step else n


def draw(rng):
    kind = rng.choice(["embed", "embed", "embed_add", "embed_palette", "loss", "loss", "loss", "norm", "norm"])
    fmt, share = rng.choice(["bf16", "fp16"]), rng.choice([0.0, 0.02, 0.25])
    index = rng.choice(["int64", "int64", "int32"])
    if kind == "norm":
        m, n = _log(rng, 1, 65536), _size(rng, 64, 16384)
        while m * n > 8192 * 8192:
            m //= 2
        c = _norm("", m, n, fmt=fmt, train=rng.random() < 0.7, post=rng.random() < 0.5,
                  gate=rng.choice(["none", "vector", "matrix"]), scale=rng.choice([1.0, 0.5, 0.25]))
    elif kind == "loss":
        m, n, k = _log(rng, 1, 8192), _size(rng, 200, 131072), _size(rng, 64, 8192)
        while m * n * k > _MOST or m * n > 8192 * 40000:
            m //= 2
        c = _loss("", m, n, k, fmt=fmt, index=index, train=rng.random() < 0.6, reduction=rng.choice(["none", "sum", "mean", "mean"]),
                  share=share)
    else:
        m, v, d = _log(rng, 1, 131072), _size(rng, 200, 131072), _size(rng, 64, 8192)
        while m * d > 65536 * 4096:
            m //= 2
        while v * d > 65536 * 4096:
            v //= 2
        c = _embed("", kind, m, v, d, fmt=fmt, index=index, scale=rng.choice([1.0, 0.5, 64.0]), share=share)
        if kind == "embed_palette":
            c["bits"] = rng.randint(1, 4)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs


def _gen(seed, i):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000 * seed + i)
    return gen


def _randn(seed, i, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed, i), device="cuda") * scale).to(dtype)


def _tokens(case, seed, words):
    """Token i with a frequency of about 1 / i, and a share of none."""
    u = torch.rand(case["m"], generator=_gen(seed, 7), device="cuda", dtype=torch.float64)
    t = (torch.exp(u * math.log(words + 1)) - 1).long().clamp_(0, words - 1)
    none = torch.rand(case["m"], generator=_gen(seed, 8), device="cuda") < case["share"]
    return torch.where(none, torch.full_like(t, OUTSIDE), t).to(INDEX[case["index"]])


def _palette(count, b, seed):
    """Packed nearest-entry indices of N(0, 0.02^2) weights, and the table: the
    middles of 2^b equally full ranges."""
    w = _randn(seed, 0, count, torch.float32, 0.02)
    part = w[:200_000].sort().values
    lut = part[((2 * torch.arange(1 << b) + 1) * part.numel() // (2 << b)).to("cuda")].contiguous()
    idx = torch.bucketize(w, (lut[1:] + lut[:-1]) / 2)
    idx = torch.nn.functional.pad(idx, (0, -idx.numel() % 8)).view(-1, 8)
    word = (idx << (b * torch.arange(8, device="cuda"))).sum(1)
    by = (word[:, None] >> (8 * torch.arange(b, device="cuda"))) & 255
    return by.to(torch.uint8).view(-1)[: (count * b + 7) // 8].contiguous(), lut


def prepare(case, seed):
    kind, t = case["kind"], DTYPES[case["fmt"]]
    s = dict(case=case)
    if kind == "norm":
        m, n, train = case["m"], case["n"], case["train"]
        s["r"] = _randn(seed, 0, (m, n), t, 2.0).requires_grad_(train)
        s["u"] = _randn(seed, 1, (m, n), t).requires_grad_(train)
        s["w"] = (1 + _randn(seed, 2, n, torch.float32, 0.2)).to(t).requires_grad_(train)
        if case["post"]:
            s["post"] = (1 + _randn(seed, 3, n, torch.float32, 0.2)).to(t).requires_grad_(train)
        if case["gate"] != "none":
            s["gate"] = _randn(seed, 4, n if case["gate"] == "vector" else (m, n), t, 0.5).requires_grad_(train)
        if train:
            s["dh"], s["dy"] = _randn(seed, 5, (m, n), t), _randn(seed, 6, (m, n), t)
        return s
    if kind == "loss":
        m, n, k, train = case["m"], case["n"], case["k"], case["train"]
        s["w"] = _randn(seed, 0, (n, k), t, 0.02)
        s["targets"] = _tokens(case, seed, n)
        # a model that has learnt something: its targets' logits stand out
        x = _randn(seed, 1, (m, k), torch.float32) + s["w"][s["targets"].long().clamp_min(0)].float() * (5.0 / (0.02 ** 2 * k))
        s["x"] = x.to(t).requires_grad_(train)
        s["w"].requires_grad_(train)
        # fp16 gradients come from a scaled loss
        up = 1024.0 if case["fmt"] == "fp16" else 1.0
        if train and case["reduction"] == "none":
            s["dloss"] = torch.rand(m, generator=_gen(seed, 2), device="cuda") * (up / m)
        elif train and case["reduction"] == "mean":
            s["dloss"] = torch.full((), up, device="cuda")
        return s
    m, v, d = case["m"], case["v"], case["d"]
    s["ids"] = _tokens(case, seed, v)
    if kind == "embed_palette":
        s["indices"], s["lut"] = _palette(v * d, case["bits"], seed)
        return s
    s["dy"] = _randn(seed, 2, (m, d), t, 0.01)
    if kind == "embed_add":
        s["grad"] = _randn(seed, 0, (v, d), t, 0.05)
    else:
        s["table"] = _randn(seed, 0, (v, d), t, 0.02).requires_grad_(True)
    return s


# ---------------------------------------------------------------------------
# the framework's operators


def _run_own(s):
    from paper_2309_00964_amd import edkm, function
    case = s["case"]
    kind = case["kind"]
    if kind == "embed_palette":
        return function.palette_embedding(s["ids"], s["indices"], s["lut"], case["v"], case["d"], case["scale"], DTYPES[case["fmt"]])
    if kind == "embed_add":
        edkm.embedding_backward(s["ids"], s["dy"], s["grad"], case["scale"], accumulate=True)
        return s["grad"]
    if kind == "embed":
        y = function.embedding(s["ids"], s["table"], case["scale"])
        return dict(y=y.detach(), grad_table=torch.autograd.grad(y, s["table"], s["dy"])[0])
    if kind == "loss":
        loss = function.linear_cross_entropy(s["x"], s["w"], s["targets"], case["reduction"])
        if not case["train"]:
            return loss
        gx, gw = torch.autograd.grad(loss, [s["x"], s["w"]], s.get("dloss"))
        return dict(loss=loss.detach(), grad_x=gx, grad_w=gw)
    h, y = function.residual_norm(s["r"], s["u"], s["w"], s.get("post"), s.get("gate"), case["scale"], EPS)
    out = dict(h=h.detach(), y=y.detach())
    if case["train"]:
        names = [x for x in ("r", "u", "w", "post", "gate") if x in s]
        g = torch.autograd.grad([h, y], [s[x] for x in names], [s["dh"], s["dy"]])
        out.update({"grad_" + x: q for x, q in zip(names, g)})
    return out


# ---------------------------------------------------------------------------
# the plain form


def _unpack(indices, at, b):
    """The b-bit indices at places `at`."""
    bit = at * b
    word = indices[bit >> 3].to(torch.int32) | (indices[(bit + b - 1) >> 3].to(torch.int32) << 8)
    return (word >> (bit & 7)) & ((1 << b) - 1)


def _embed_plain(s):
    case, t = s["case"], DTYPES[s["case"]["fmt"]]
    v, d = case["v"], case["d"]
    ids = s["ids"].long()
    there = ((ids >= 0) & (ids < v))[:, None]
    row = ids.clamp(0, v - 1)
    if case["kind"] == "embed_palette":
        at = row[:, None] * d + torch.arange(d, device=row.device)
        y = s["lut"].to(t)[_unpack(s["indices"], at, case["bits"]).long()].float()
        return (torch.where(there, y, 0.0) * case["scale"]).to(t)
    g = torch.zeros(v, d, device=row.device)
    g.index_add_(0, row, torch.where(there, s["dy"].float(), 0.0))
    g *= case["scale"]
    if case["kind"] == "embed_add":
        return s["grad"].copy_(s["grad"].float() + g)
    y = torch.where(there, s["table"].detach()[row].float(), 0.0) * case["scale"]
    return dict(y=y.to(t), grad_table=g.to(t))


def _loss_plain(s):
    case, t = s["case"], DTYPES[s["case"]["fmt"]]
    n = case["n"]
    x, w, ids = s["x"].detach().float(), s["w"].detach().float(), s["targets"].long()
    there = (ids >= 0) & (ids < n)
    col = ids.clamp(0, n - 1)[:, None]
    z = x @ w.t()
    top = z.max(1, keepdim=True).values
    at = z.gather(1, col) - top
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    loss = torch.where(there, (torch.log(total) - at)[:, 0], 0.0)
    count = there.sum().clamp_min(1)
    if case["reduction"] != "none":
        loss = loss.sum()
        if case["reduction"] == "mean":
            loss = loss / count
    if not case["train"]:
        return loss
    g = s.get("dloss", torch.ones((), device=x.device)) / (count if case["reduction"] == "mean" else 1)
    dz = (e / total).scatter_add_(1, col, torch.full_like(at, -1.0)) * torch.where(there, g, 0.0)[:, None]
    return dict(loss=loss, grad_x=(dz @ w).to(t), grad_w=(dz.t() @ x).to(t))


def _rms(v):
    return torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)


def _norm_plain(s):
    case, t = s["case"], DTYPES[s["case"]["fmt"]]
    a = case["scale"]
    r, u, w = (s[x].detach().float() for x in ("r", "u", "w"))
    post = s["post"].detach().float() if case["post"] else None
    gate = s["gate"].detach().float() if case["gate"] != "none" else 1.0
    su = _rms(u) if case["post"] else None
    b = u * su * post if case["post"] else u
    h = r + a * gate * b
    sh = _rms(h)
    hn = h * sh
    out = dict(h=h.to(t), y=(hn * w).to(t))
    if not case["train"]:
        return out
    dy, dh = s["dy"].float(), s["dh"].float()
    g = dy * w
    dh = dh + sh * (g - hn * (g * hn).mean(1, keepdim=True))
    out.update(grad_r=dh.to(t), grad_w=(dy * hn).sum(0).to(t))
    q = a * gate * dh
    if case["post"]:
        un = u * su
        out["grad_post"] = (q * un).sum(0).to(t)
        q = q * post
        q = su * (q - un * (q * un).mean(1, keepdim=True))
    out["grad_u"] = q.to(t)
    if case["gate"] != "none":
        dg = a * dh * b
        out["grad_gate"] = (dg.sum(0) if case["gate"] == "vector" else dg).to(t)
    return out


def _run_plain(s):
    kind = s["case"]["kind"]
    return _loss_plain(s) if kind == "loss" else _norm_plain(s) if kind == "norm" else _embed_plain(s)


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---------------------------------------------------------------------------


def work(case):
    kind, m = case["kind"], case["m"]
    if kind == "norm":
        n = case["n"]
        one = 2 * m * n
        vectors = 2 * n * (1 + case["post"] + (case["gate"] == "vector"))
        gate = one * (case["gate"] == "matrix")
        b = 4 * one + gate + vectors
        if case["train"]:      # dh, dy; dr, du and the gate's; the vectors' gradients
            b += 4 * one + gate + vectors
        return {"bytes": b, "flops": (30 if case["train"] else 10) * m * n}
    if kind == "loss":
        n, k = case["n"], case["k"]
        b = 2 * (m * k + n * k) + 12 * m
        return {"bytes": 2 * b if case["train"] else b, "flops": (6 if case["train"] else 2) * m * n * k}
    v, d, i = case["v"], case["d"], 8 if case["index"] == "int64" else 4
    rows = min(m, v)
    if kind == "embed_palette":
        return {"bytes": m * i + rows * d * case["bits"] / 8 + 2 * m * d, "flops": m * d}
    if kind == "embed_add":
        return {"bytes": m * i + 2 * m * d + 4 * rows * d, "flops": 2 * m * d}
    return {"bytes": m * i + 2 * rows * d + 4 * m * d + 2 * v * d, "flops": 3 * m * d}


def exact(case, seed):
    """The same results in 64 bits."""
    s = prepare(case, seed)
    kind, t = case["kind"], DTYPES[case["fmt"]]
    if kind == "norm":
        x = {name: s[name].detach().double().requires_grad_(case["train"]) for name in ("r", "u", "w", "post", "gate") if name in s}

        def norm(v, w):
            return v / torch.sqrt(v.pow(2).sum(-1, keepdim=True) / case["n"] + EPS) * w
        b = norm(x["u"], x["post"]) if case["post"] else x["u"]
        h = x["r"] + (x["gate"] * b if "gate" in x else b) * case["scale"]
        y = norm(h, x["w"])
        out = dict(h=h.detach(), y=y.detach())
        if case["train"]:
            g = torch.autograd.grad([h, y], list(x.values()), [s["dh"].double(), s["dy"].double()])
            out.update({"grad_" + name: q for name, q in zip(x, g)})
        return out
    if kind == "loss":
        m, n = case["m"], case["n"]
        w, ids = s["w"].detach().double(), s["targets"].long()
        there = (ids >= 0) & (ids < n)
        weight = there.double()
        if case["reduction"] == "mean":
            weight = weight / max(1, int(there.sum()))
        weight = weight * s.get("dloss", torch.ones((), device=w.device)).double()
        losses, gx, gw = [], [], torch.zeros_like(w)
        step = max(1, (1 << 27) // n)
        for a in range(0, m, step):
            x = s["x"].detach()[a:a + step].double()
            lp = torch.log_softmax(x @ w.t(), 1)
            part = there[a:a + step]
            rows = torch.arange(x.shape[0], device=x.device)[part]
            one = torch.zeros(x.shape[0], dtype=torch.float64, device=x.device)
            one[part] = -lp[rows, ids[a:a + step][part]]
            losses.append(one)
            if case["train"]:
                p = lp.exp_()
                p[rows, ids[a:a + step][part]] -= 1
                p *= weight[a:a + step, None]
                gx.append(p @ w)
                gw += p.t().contiguous() @ x
        loss = torch.cat(losses)
        if case["reduction"] != "none":
            loss = loss.sum() / (max(1, int(there.sum())) if case["reduction"] == "mean" else 1)
        return dict(loss=loss, grad_x=torch.cat(gx), grad_w=gw) if case["train"] else loss
    m, v, d = case["m"], case["v"], case["d"]
    ids = s["ids"].long()
    part = (ids >= 0) & (ids < v)
    if kind == "embed_palette":
        # the stream's bits one by one
        at = (ids[part, None] * d + torch.arange(d, device=ids.device)) * case["bits"]
        idx = torch.zeros_like(at)
        for j in range(case["bits"]):
            idx |= ((s["indices"][(at + j) >> 3].to(torch.int64) >> ((at + j) & 7)) & 1) << j
        y = torch.zeros(m, d, dtype=torch.float64, device=ids.device)
        y[part] = s["lut"].to(t).double()[idx] * case["scale"]
        return y
    g = torch.zeros(v, d, dtype=torch.float64, device=ids.device)
    g.index_add_(0, ids[part], s["dy"][part].double() * case["scale"])
    if kind == "embed_add":
        return g + s["grad"].double()
    y = torch.zeros(m, d, dtype=torch.float64, device=ids.device)
    y[part] = s["table"].detach().double()[ids[part]] * case["scale"]
    return dict(y=y, grad_table=g)
