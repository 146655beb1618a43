"""Products and AdamW steps in plain 64-bit torch, and bounds on what fp32 sums and
16-bit roundings may add to them — test infrastructure only."""
import math

import numpy as np
import torch

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "gelu", "silu")
# |act'| and |act''| at most: gelu' peaks at 1.129 (z = sqrt 2), silu' at 1.0999; gelu'' at
# 2 phi(0) = 0.798, silu'' at 1/2
SLOPE = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "silu": 1.1}
CURVE = {"none": 0.0, "relu": 0.0, "gelu": 0.8, "silu": 0.5}


def half(dtype):
    """Half a step, relative."""
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half a subnormal step: what rounding may add to a value near 0."""
    f = torch.finfo(dtype)
    return f.smallest_normal * f.eps / 2


def act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if name == "silu":
        q = torch.sigmoid(z)
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def product(x, w, bias, residual, name):
    """z, y and the bound of y's error: a sum of d products in fp32, whatever its order,
    is off by at most (d + 2) 2^-23 of the sum of magnitudes (every addition by an ulp);
    the activation's own fp32 formula by a few ulps of its argument and value; then one
    rounding."""
    d = x.shape[1]
    z = x.double() @ w.double().t()
    mag = x.double().abs() @ w.double().abs().t()
    if bias is not None:
        z = z + bias.double()
        mag = mag + bias.double().abs()
    a = act(z, name)
    y = a if residual is None else a + residual.double()
    err = (d + 2) * 2.0 ** -23 * mag * SLOPE[name] + 2.0 ** -20 * (z.abs() + a.abs()) + 2.0 ** -23 * y.abs()
    return z, y, y.abs() * half(x.dtype) + tiny(x.dtype) + err * (1 + half(x.dtype))


def gradients(dy, x, w, z, name):
    """dx, dw, db with their bounds.  The kept z is off by its rounding (and the fp32 sum's
    error, smaller than that step for every size here), which moves dz by |dy act''| of it;
    dz is rounded once more on the way into the products."""
    h, t = half(x.dtype), tiny(x.dtype)
    m, n = dy.shape
    dy, x, w = dy.double(), x.double(), w.double()
    if z is None:            # without activation it is not looked at
        z = torch.zeros_like(dy)
    dz = dy * slope(z, name)
    e0 = dy.abs() * (CURVE[name] * (2 * h * z.abs() + t + 2.0 ** -20) + 2.0 ** -20 * (name != "none"))
    if name == "relu":       # within z's error of 0 the slope is one side's or the other's
        e0 = e0 + dy.abs() * (z.abs() <= 2.0 ** -16)
    e1 = e0 + ((dz.abs() + e0) * h + t if name != "none" else 0)
    out = {}
    for key, val, mag, e, d in (
            ("dx", dz @ w, dz.abs() @ w.abs(), e1 @ w.abs(), n),
            ("dw", dz.t() @ x, dz.abs().t() @ x.abs(), e1.t() @ x.abs(), m),
            ("db", dz.sum(0), dz.abs().sum(0), e0.sum(0), m)):
        err = e + (d + 2) * 2.0 ** -23 * (mag + e)
        out[key] = (val, val.abs() * h + t + err * (1 + h))
    return out


def assert_within(got, ref, bound, what):
    off = (got.double() - ref).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = int((off / bound).nan_to_num(nan=math.inf).argmax())
        raise AssertionError("%s: %d of %d outside; worst at %d: %r, want %r +- %r" % (
            what, int(bad.sum()), got.numel(), i, float(got.reshape(-1)[i]), float(ref.reshape(-1)[i]),
            float(bound.reshape(-1)[i])))


def palette(n, k, bits, seed):
    """Random indices and their packed stream, and a table with values of both signs."""
    from oracle import palette as pal
    rng = np.random.default_rng(seed)
    idx = rng.integers(0, 1 << bits, n * k, dtype=np.uint8)
    lut = (rng.standard_normal(1 << bits) * 0.02).astype(np.float32)
    return idx, pal.pack(idx, bits), lut


def hash32(h):
    h = h & 0xFFFFFFFF
    h ^= h >> 16
    h = (h * 0x85EBCA6B) & 0xFFFFFFFF
    h ^= h >> 13
    h = (h * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


F8 = {torch.float8_e4m3fn: (3, 7, 448.0), torch.float8_e5m2: (2, 15, 57344.0)}


def to_float8(x, step, seed, dtype):
    """Codes and block scales of an fp32 state, from the definition: the two float8
    neighbours of a value, and which of them the noise takes."""
    man, bias, top = F8[dtype]
    n = x.numel()
    xb = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
    amax = xb.abs().amax(1, keepdim=True)
    live = amax >= 2.0 ** -100
    scale = torch.where(live, amax * np.float32(1 / np.float32(top)), torch.zeros_like(amax))
    y = (xb.abs() * torch.where(live, amax.reciprocal() * top, torch.zeros_like(amax))).clamp_max(top).view(-1)[:n]
    grid = torch.arange(0, 0x7F if man == 3 else 0x7C, dtype=torch.uint8).view(dtype).float()   # ascending finite values
    low = (torch.bucketize(y, grid, right=True) - 1).clamp(0, grid.numel() - 2)
    lo, hi = grid[low].double(), grid[low + 1].double()
    i = torch.arange(n)
    pair = hash32((i >> 1) + int(step) * 0x9E3779B9 + int(seed))
    noise = torch.where(i % 2 == 1, pair >> 16, pair & 0xFFFF).double()
    code = low + ((y.double() - lo) / (hi - lo) + (noise + 0.5) / 65536 >= 1).to(low.dtype)
    if man == 2:
        code = torch.where((code == 0) & (y > 0), torch.ones_like(code), code)
    code = code | torch.where(x.signbit(), 128, 0)
    return code.to(torch.uint8), scale.view(-1)
