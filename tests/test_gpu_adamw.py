"""The AdamW step against the formula: fp32 states in 64 bits, 8-bit states bit for bit
from the definition of their rounding, many tensors at once, captured steps, and what
non-finite gradients and tiny blocks leave."""
import sys

import pytest

torch = pytest.importorskip("torch")

import layer_util as L                                             # noqa: E402
from paper_2309_00964_amd import edkm                              # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def say(*a):
    print("[gpu-case]", *a, flush=True)
    sys.stdout.flush()


def randn(gen, n, scale, dtype=torch.float32):
    return (torch.randn(n, generator=gen) * scale).to(dtype)


def blocks(n):
    return (n + 255) // 256


class Tensors:
    """Lists of one batch on the CPU and their copies on the GPU.  `lead`: elements before
    each tensor in its buffer (unaligned starts)."""

    def __init__(self, sizes, pt, gt, bits, master, seed, lead=0):
        gen = torch.Generator().manual_seed(seed)
        self.sizes, self.bits = sizes, bits
        c = {"p": [], "g": [], "m": [], "v": [], "ms": [], "vs": [], "w": []}
        for n in sizes:
            w = randn(gen, n, 0.02)
            c["w"].append(w)
            c["p"].append(w.to(TYPES[pt]))
            c["g"].append(randn(gen, n, 1e-2, TYPES[gt]))
            m, v = randn(gen, n, 3e-3), randn(gen, n, 1e-2).square()
            if bits == 8:
                for key, x, t in (("m", m, torch.float8_e4m3fn), ("v", v, torch.float8_e5m2)):
                    code, scale = L.to_float8(x, 0, 1, t)
                    c[key].append(code.view(t))
                    c[key + "s"].append(scale)
            else:
                c["m"].append(m)
                c["v"].append(v)
        self.cpu = c
        self.gpu = {k: [self.place(t, lead) for t in ts] for k, ts in c.items()}
        self.master = master
        self.step = torch.full((1,), 4, dtype=torch.int32, device=DEV)

    @staticmethod
    def place(t, lead):
        raw = torch.zeros(t.numel() + lead + 8, dtype=t.dtype).view(torch.uint8)
        buf = raw.to(DEV).view(t.dtype)
        buf.view(torch.uint8)[lead * t.element_size():(lead + t.numel()) * t.element_size()].copy_(t.view(torch.uint8))
        return buf[lead:lead + t.numel()]

    def run(self, seed=7, **kw):
        g = self.gpu
        edkm.adamw_batch(g["p"], g["g"], g["m"], g["v"], self.step, masters=g["w"] if self.master else None,
                         m_scales=g["ms"] if self.bits == 8 else None, v_scales=g["vs"] if self.bits == 8 else None,
                         seed=seed, **{**HYPER, **kw})


def moments(c, i, bits):
    m, v = c["m"][i].float(), c["v"][i].float()
    if bits == 8:
        n = m.numel()
        m = m * c["ms"][i].repeat_interleave(256)[:n]
        v = v * c["vs"][i].repeat_interleave(256)[:n]
    return m, v


def reference(T, i, t, pt):
    """m and v in the step's fp32 operations, p in 64 bits from them."""
    c, b1, b2 = T.cpu, HYPER["beta1"], HYPER["beta2"]
    m, v = moments(c, i, T.bits)
    g = c["g"][i].float()
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    p = (c["w"][i] if T.master else c["p"][i]).double()
    up = HYPER["lr"] * (m.double() / (1 - b1 ** t)) / ((v.double() / (1 - b2 ** t)).sqrt() + HYPER["eps"])
    return m, v, p - HYPER["lr"] * HYPER["weight_decay"] * p - up, up


SIZES = [1, 2, 255, 256, 257, 4095, 4097, 20_003, 70_000]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pt,gt,master", [("fp32", "fp32", False), ("bf16", "bf16", False), ("fp16", "fp32", False),
                                          ("fp16", "fp16", True), ("bf16", "fp32", True)])
@pytest.mark.parametrize("lead", [0, 1])
def test_step(bits, pt, gt, master, lead):
    say("adamw", bits, pt, gt, master, lead)
    T = Tensors(SIZES, pt, gt, bits, master, 5, lead)
    T.run()
    torch.cuda.synchronize()
    assert int(T.step) == 5
    for i, n in enumerate(T.sizes):
        m, v, p, up = reference(T, i, 5, pt)
        got = {k: ts[i].cpu() for k, ts in T.gpu.items() if i < len(ts)}
        # p: three fp32 roundings of |p|-sized numbers and about 8 ulps of the update
        tol = 3 * 2.0 ** -24 * p.abs() + 8 * 2.0 ** -23 * up.abs()
        if master:
            L.assert_within(got["w"], p, tol, "master %d" % n)
            assert torch.equal(got["p"], got["w"].to(TYPES[pt]))
        else:
            d = TYPES[pt]
            L.assert_within(got["p"], p, tol + (p.abs() * L.half(d) * (1 + 2.0 ** -20) + L.tiny(d) if pt != "fp32" else 0), "p %d" % n)
        if bits == 8:
            for key, x, t in (("m", m, torch.float8_e4m3fn), ("v", v, torch.float8_e5m2)):
                code, scale = L.to_float8(x, 5, 7, t)
                assert torch.equal(got[key + "s"], scale), (key, n)
                assert torch.equal(got[key].view(torch.uint8), code), (key, n)
        else:
            assert torch.equal(got["m"], m) and torch.equal(got["v"], v), n


def test_many_tensors_are_their_single_steps():
    sizes = [1 + 37 * (i % 11) for i in range(70)]       # three launches
    say("many tensors")
    A, B = (Tensors(sizes, "bf16", "bf16", 8, True, 9) for _ in range(2))
    A.run()
    g = B.gpu
    for i in range(len(sizes)):
        step = torch.full((1,), 4, dtype=torch.int32, device=DEV)
        edkm.adamw_batch([g["p"][i]], [g["g"][i]], [g["m"][i]], [g["v"][i]], step, masters=[g["w"][i]], m_scales=[g["ms"][i]],
                         v_scales=[g["vs"][i]], seed=7, **HYPER)
    for k in A.gpu:
        for a, b in zip(A.gpu[k], g[k]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), k


def test_empty_tensors_and_rate_on_the_device():
    say("empty tensors, lr tensor")
    A, B = (Tensors([0, 300, 0, 5], "fp16", "fp16", 32, True, 11) for _ in range(2))
    A.run()
    B.run(lr=torch.full((1,), HYPER["lr"], device=DEV))
    assert int(A.step) == 5 and int(B.step) == 5
    for a, b in zip(A.gpu["w"], B.gpu["w"]):
        # the rate is fp32 on the device and fp64 here: the decay factor may differ by an ulp
        torch.testing.assert_close(a, b, rtol=2.0 ** -21, atol=1e-9)


def test_small_increments_are_kept_on_average():
    """A second moment that decays by 0.1% a step moves by that on average although a
    float8 step is 25%: the noise carries it.  Over n elements the mean's deviation is at
    most 6 sigma of a 25%-step coin."""
    n, b2 = 1 << 20, 0.999
    say("noise keeps small increments")
    g = torch.zeros(n, device=DEV)
    m, v = torch.zeros(n, device=DEV).to(torch.float8_e4m3fn), torch.full((n,), 40000.0, device=DEV)
    v[::256] = 57344.0
    v = v.to(torch.float8_e5m2)
    before = v.float().mean().item()
    ms, vs = torch.zeros(n // 256, device=DEV), torch.full((n // 256,), 1e-6, device=DEV)
    step = torch.zeros(1, dtype=torch.int32, device=DEV)
    p = torch.zeros(n, device=DEV)
    for _ in range(20):
        edkm.adamw_batch([p], [g], [m], [v], step, 0.0, 0.9, b2, m_scales=[ms], v_scales=[vs], seed=3)
    mean = (v.float().view(-1, 256) * vs[:, None]).mean().item()
    want = before * 1e-6 * b2 ** 20
    assert abs(mean - want) <= want * (6 * 0.25 * (20 ** 0.5) / n ** 0.5 + 1e-5)


def test_non_finite_and_tiny_gradients():
    n = 1024
    for bits in (32, 8):
        say("non-finite gradients", bits)
        T = Tensors([n], "fp32", "fp32", bits, False, 13)
        T.gpu["g"][0][300] = float("nan")
        T.gpu["g"][0][600] = float("inf")
        before = T.gpu["p"][0].clone()
        T.run()
        p = T.gpu["p"][0]
        assert p.isnan().nonzero().flatten().tolist() == [300, 600]
        assert not torch.equal(p[:300], before[:300])
        m, v = T.gpu["m"][0].float(), T.gpu["v"][0].float()
        if bits == 8:
            m, v = (x * T.gpu[s][0].repeat_interleave(256) for x, s in ((m, "ms"), (v, "vs")))
            for x in (m, v):
                assert bool(x[256:768].isnan().all()) and bool(x[:256].isfinite().all()) and bool(x[768:].isfinite().all())
        else:
            assert m[300].isnan() and v[600] == float("inf") and int(m.isfinite().sum()) == n - 2
    say("zeros and tiny blocks")
    z = lambda t=torch.float32: torch.zeros(512, device=DEV).to(t)  # noqa: E731
    p, g = torch.ones(512, device=DEV), z()
    g[256:] = 1e-25                       # g^2 is below 2^-100, m is not
    m, v, ms, vs = z(torch.float8_e4m3fn), z(torch.float8_e5m2), torch.ones(2, device=DEV), torch.ones(2, device=DEV)
    step = torch.zeros(1, dtype=torch.int32, device=DEV)
    edkm.adamw_batch([p], [g], [m], [v], step, 1e-3, weight_decay=0.0, m_scales=[ms], v_scales=[vs])
    assert ms[0] == 0 and vs.tolist() == [0, 0] and ms[1] > 0
    assert not bool(v.float().any()) and bool((p == 1).all())
    assert bool((m[256:].float() == 448).all())


def test_second_moment_never_becomes_zero():
    """Elements 2^-14 of the block's largest gradient: their v is far below the smallest
    float8 number, and is stored as that."""
    say("small v")
    g = torch.full((256,), 2.0 ** -20, device=DEV)
    g[0] = 1.0
    z = lambda t: torch.zeros(256, device=DEV).to(t)  # noqa: E731
    m, v, s = z(torch.float8_e4m3fn), z(torch.float8_e5m2), [torch.zeros(1, device=DEV) for _ in range(2)]
    p, step = torch.zeros(256, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    edkm.adamw_batch([p], [g], [m], [v], step, 1e-3, m_scales=[s[0]], v_scales=[s[1]])
    assert bool((v.view(torch.uint8)[1:] == 1).all()) and v.view(torch.uint8)[0] == 0x7B


def test_captured_and_replayed():
    say("graph")
    A, B = (Tensors([3000, 77], "bf16", "bf16", 8, True, 17) for _ in range(2))
    A.run()
    B.run()
    torch.cuda.synchronize()
    lr = torch.full((1,), 1e-3, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.run(lr=lr)
    for i in range(3):
        lr.fill_(1e-3 * (i + 1))
        for T in (A, B):
            for g in T.gpu["g"]:
                g.mul_(-0.5)
        graph.replay()
        B.run(lr=lr)
        torch.cuda.synchronize()
        assert int(A.step) == int(B.step) == 6 + i
        for k in A.gpu:
            for a, b in zip(A.gpu[k], B.gpu[k]):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (i, k)
