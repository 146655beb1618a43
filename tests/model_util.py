"""The operators at a model's ends and between its blocks in plain 64-bit torch, with bounds
on what fp32 sums and 16-bit roundings may add to them — test infrastructure only."""
import torch

from layer_util import half, tiny

U = 2.0 ** -23        # an fp32 operation is off by at most an ulp of this, relative


def rounded(ref, err, dtype):
    """Bound of a value that is off by `err` before its one rounding to `dtype`."""
    return ref.abs() * half(dtype) + tiny(dtype) + err * (1 + 2 * half(dtype))


def embedding(ids, table, scale):
    """y and its bound: a product in fp32, rounded once."""
    v = table.shape[0]
    there = (ids >= 0) & (ids < v)
    y = torch.where(there[:, None], table.double()[ids.long().clamp(0, v - 1)], 0.0) * scale
    return y, rounded(y, y.abs() * U, table.dtype)


def embedding_grad(ids, dy, v, scale, old=None):
    """dtable and its bound: a sum of c values in fp32, in any order, is off by at most c ulps
    of the sum of magnitudes; the scaled addition by one more of the result."""
    part = (ids >= 0) & (ids < v)
    at, g = ids.long()[part], dy.double()[part]
    zero = torch.zeros(v, dy.shape[1], dtype=torch.float64, device=dy.device)
    s, mag = zero.index_add(0, at, g) * scale, zero.index_add(0, at, g.abs()) * abs(scale)
    count = torch.zeros(v, dtype=torch.float64, device=dy.device).index_add(0, at, torch.ones_like(at, dtype=torch.float64))
    ref = s if old is None else old.double() + s
    err = (count[:, None] + 1) * U * mag + U * ref.abs()
    return ref, rounded(ref, err, dy.dtype)


def norm(v, w, eps):
    s = 1 / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + eps)
    return v * s * w


def residual_norm(r, u, w, post, gate, scale, eps):
    """h, y and their bounds.  A mean of n squares is off by (n + 2) ulps relative, its root by
    half of that; the reciprocal root and each product by an ulp or two."""
    dt, n = r.dtype, r.shape[1]
    d = [None if t is None else t.double() for t in (r, u, w, post, gate)]
    r, u, w, post, gate = d
    root = ((n + 2) / 2 + 4) * U
    if u is None:
        h, eh = r, torch.zeros_like(r)
    else:
        b = u if post is None else norm(u, post, eps)
        b = b * scale if gate is None else b * gate * scale
        h = r + b
        eh = b.abs() * (3 + (0 if post is None else 1)) * U + (b.abs() * root if post is not None else 0) + h.abs() * U
    y = norm(h, w, eps)
    s = 1 / torch.sqrt(h.pow(2).mean(-1, keepdim=True) + eps)
    # h's error moves y by itself, and through the row's root by at most the root of its mean square
    ey = (eh + h.abs() * s * eh.pow(2).mean(-1, keepdim=True).sqrt()) * s * w.abs() * (1 + root) + y.abs() * (root + 3 * U)
    return h, y, rounded(h, eh, dt), rounded(y, ey, dt)


def residual_norm_grads(dy, dh, r, u, w, post, gate, scale, eps):
    """The gradients and their bounds, term by term."""
    dt, (m, n) = r.dtype, r.shape
    z = torch.zeros(m, n, dtype=torch.float64, device=r.device)
    dy = z if dy is None else dy.double()
    dh = z if dh is None else dh.double()
    w = w.double()
    root = ((n + 2) / 2 + 4) * U

    def back(v, ev, g, wt):
        """Through N(v; wt) for the gradient g, v being off by ev: dv and the bound of its fp32
        error, the normed v and its own."""
        s = 1 / torch.sqrt(v.pow(2).mean(1, keepdim=True) + eps)
        vn, gw = v * s, g * wt
        rel = s * ev.pow(2).mean(1, keepdim=True).sqrt()        # of the root, by v's error
        en = s * ev + vn.abs() * (rel + root + 2 * U)
        mean, mag = (gw * vn).mean(1, keepdim=True), (gw * vn).abs().mean(1, keepdim=True)
        em = (gw.abs() * en).mean(1, keepdim=True) + mag * (n + 6) * U
        dv = s * (gw - vn * mean)
        err = s * (gw.abs() * (rel + root + 4 * U) + vn.abs() * em + en * (mag + em) + (vn * mean).abs() * (rel + root + 4 * U))
        return dv, err, vn, en, s

    h = r.double()
    eh = torch.zeros_like(h)
    if u is not None:
        # h in fp32, as in residual_norm
        b = u.double() if post is None else norm(u.double(), post.double(), eps)
        b = b * scale if gate is None else b * gate.double() * scale
        h = h + b
        eh = b.abs() * 4 * U + (b.abs() * root if post is not None else 0) + h.abs() * U
    dv, err, hn, en, _ = back(h, eh, dy, w)
    d = dh + dv
    ed = err + d.abs() * U
    out = {"dr": (d, rounded(d, ed, dt))}

    def column(val, e):
        ref = val.sum(0)
        bound = e.sum(0) + (m + 2) * U * (val.abs() + e).sum(0)
        return ref, rounded(ref, bound, dt)

    out["dw"] = column(dy * hn, dy.abs() * en + (dy * hn).abs() * U)
    if u is None:
        return out
    u = u.double()
    g = scale if gate is None else scale * gate.double()
    ag = abs(scale) if gate is None else abs(scale) * gate.double().abs()
    q, eq = d * g, ed * ag + (d * g).abs() * 2 * U
    if post is None:
        out["du"] = (q, rounded(q, eq, dt))
        b, eb = u, torch.zeros_like(u)
    else:
        p = post.double()
        du, eu, un, _, s = back(u, torch.zeros_like(u), q, p)
        # q's own error goes through the same linear map
        eu = eu + s * (eq * p.abs() + un.abs() * (eq * p.abs() * un.abs()).mean(1, keepdim=True)) * (1 + 4 * root)
        out["du"] = (du, rounded(du, eu, dt))
        out["dpost"] = column(q * un, eq * un.abs() + (q * un).abs() * (root + 3 * U))
        b, eb = un * p, (un * p).abs() * (root + 2 * U)
    if gate is not None:
        dg, eg = scale * d * b, abs(scale) * (ed * b.abs() + d.abs() * eb) + (scale * d * b).abs() * 4 * U
        out["dgate"] = (dg, rounded(dg, eg, dt)) if gate.dim() == 2 else column(dg, eg)
    return out


def cross_entropy(x, w, targets, reduction):
    """loss, lse, and their bounds.  A logit is a sum of k products in fp32 (off by (k + 2) ulps
    of the sum of magnitudes); e^(z - top) then by that and an ulp of z - top, relative, and the sum's
    logarithm by the largest such error and (n + 20) ulps for the sum itself."""
    n, k = w.shape
    z, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    ez = (k + 2) * U * mag.amax(1)
    there = (targets >= 0) & (targets < n)
    lse = torch.logsumexp(z, 1)
    span = (z.amax(1, keepdim=True) - z).clamp_max(104).amax(1)     # beyond it e^ is 0 in fp32
    e_lse = ez + (n + 20 + 4 * span) * U + 2 * U * lse.abs()
    loss = torch.where(there, lse - z.gather(1, targets.long().clamp(0, n - 1)[:, None])[:, 0], 0.0)
    e = torch.where(there, e_lse + ez + 2 * U * (z.amax(1).abs() + loss.abs()) + 2 * U * z.abs().amax(1), 0.0)
    lse, e_lse = torch.where(there, lse, 0.0), torch.where(there, e_lse, 0.0)
    if reduction == "none":
        return loss, e + tiny(torch.float32), lse, e_lse + tiny(torch.float32)
    count = int(there.sum())
    total = loss.sum()
    over = max(1, count) if reduction == "mean" else 1
    bound = (e.sum() + (count + 4) * U * loss.abs().sum()) / over + U * total.abs() / over
    return total / over, bound + tiny(torch.float32), lse, e_lse + tiny(torch.float32)


def cross_entropy_grads(dloss, x, w, targets, reduction):
    """dx, dw and their bounds.  dz is rounded once to 16 bits as a share of 2^15 times the
    largest |g| (so a subnormal step is that much smaller), each product summed in fp32."""
    dt = x.dtype
    n, k = w.shape
    z, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    there = (targets >= 0) & (targets < n)
    g = dloss.double().expand(x.shape[0]) / (max(1, int(there.sum())) if reduction == "mean" else 1)
    g = torch.where(there, g, 0.0)[:, None]
    p = torch.softmax(z, 1)
    ez = (k + 2) * U * mag.amax(1, keepdim=True)
    ep = p * (2 * ez + (n + 40 + 8 * z.abs().amax(1, keepdim=True)) * U)
    one = torch.zeros_like(p).scatter_(1, targets.long().clamp(0, n - 1)[:, None], 1.0)
    dz = g * (p - one)
    e0 = g.abs() * (ep + 2 * U)
    ed = e0 + (dz.abs() + e0) * half(dt) + tiny(dt) * g.abs().max() / 2 ** 15 + dz.abs() * 4 * U
    ed = torch.where(g == 0, 0.0, ed)
    xs = torch.where(g == 0, 0.0, x.double())
    out = {}
    for key, a, e, b, depth in (("dx", dz, ed, w.double(), n), ("dw", dz.t().contiguous(), ed.t().contiguous(), xs, x.shape[0])):
        val, m = a @ b, a.abs() @ b.abs()
        err = e @ b.abs()
        err = err + (depth + 4) * U * (m + err)
        out[key] = (val, rounded(val, err, dt))
    return out
