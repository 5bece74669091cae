"""Injection between two norms, forward and gradients, against the formulas in 64 bits."""
import math
import os
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def formula(h, m, wp, wn, gate, sigmoid, lam, eps):
    s = torch.ones((), dtype=torch.float64)
    if gate is not None:
        s = gate[:, None] if gate.dim() == 1 else gate
        s = torch.sigmoid(s) if sigmoid else s
    u = h + lam * s * (wp * m / torch.sqrt((m * m).mean(1, keepdim=True) + eps))
    return u, wn * u / torch.sqrt((u * u).mean(1, keepdim=True) + eps)


def make(seed, n, d, kind, gate, weights="f32", zero_row=True):
    rng = torch.Generator().manual_seed(seed)
    h = torch.randn((n, d), generator=rng).to(TYPES[kind])
    m = (torch.randn((n, d), generator=rng) * 0.1).to(TYPES[kind])
    if zero_row and n > 1:
        m[n // 2] = 0
    g = {"none": None, "scalar": torch.randn(n, generator=rng), "vector": torch.randn((n, d), generator=rng).to(TYPES[kind])}[gate]
    wp, wn = ((1 + 0.3 * torch.randn(d, generator=rng)).to(TYPES[weights]) for _ in range(2))
    gu, gn = (torch.randn((n, d), generator=rng).to(TYPES[kind]) for _ in range(2))
    return h, m, wp, wn, g, gu, gn


def near(got, want, tol, what):
    """tol: the error of the sums and products in 32 bits, elementwise; the result's own rounding is added."""
    got = got.double().cpu()
    off = (got - want).abs()
    allowed = tol + HALF[torch.bfloat16 if what.endswith("bf16") else torch.float32] * (want.abs() + tol)
    assert bool((off <= allowed + 1e-37).all()), (what, float((off - allowed).max()), float(off.max()))


def check(data, sigmoid=False, lam=0.75, eps=1e-6, move=lambda x: None if x is None else x.to(DEV)):
    """A sum over a row of d terms is off by at most (d / 8 / 32 + 18) 2^-24 of its magnitudes (chains of 8, then shuffles and up to 32
    partial sums); each result is a handful of factors, each rounded once (2^-24) or twice, an exponential 2^-21.  So every term of a
    result is off by at most R = 2^-18 of its magnitude for rows up to 8192; terms that cancel are taken by their magnitudes."""
    from paper_2607_07388_b200 import engine
    h, m, wp, wn, g, gu, gn = data
    dev = [move(x) for x in data]
    kw = dict(sigmoid=sigmoid, lam=lam, eps=eps)
    out, normed = engine.normed_inject_forward(*dev[:5], **kw)
    grads = engine.normed_inject_backward(dev[5], dev[6], *dev[:5], **kw)
    leaves = [None if x is None else x.double().requires_grad_() for x in (h, m, wp, wn, g)]
    u, normed_e = formula(*leaves, sigmoid, lam, eps)
    torch.autograd.backward([u, normed_e], [gu.double(), gn.double()])
    R, D = 2.0 ** -18, "bf16" if h.dtype == torch.bfloat16 else "f32"
    W = "bf16" if wp.dtype == torch.bfloat16 else "f32"
    with torch.no_grad():
        H, M, P, N = (x.abs() for x in leaves[:4])
        s = torch.ones((), dtype=torch.float64) if g is None else (leaves[4][:, None] if g.dim() == 1 else leaves[4])
        s = torch.sigmoid(s) if sigmoid and g is not None else s.abs()
        a = 1 / torch.sqrt((M * M).mean(1, keepdim=True) + eps)
        y = a * M * P
        um = H + abs(lam) * s * y
        b = 1 / torch.sqrt((u * u).mean(1, keepdim=True) + eps)
        # u's own error reaches b through u u
        slack = 1 + (um * um).mean(1, keepdim=True) * b * b
        near(out, u.detach(), R * um, f"out {D}")
        near(normed, normed_e.detach(), R * N * um * b * slack, f"normed {D}")
        t = N * gn.double().abs()
        du = gu.double().abs() + b * t + um * b ** 3 * (um * t).mean(1, keepdim=True)
        du = du * slack
        dy = abs(lam) * s * du
        x = P * dy
        near(grads[0], leaves[0].grad, R * du, f"grad_h {D}")
        near(grads[1], leaves[1].grad, R * (a * x + M * a ** 3 * (M * x).mean(1, keepdim=True)), f"grad_m {D}")
        rows = 1 + len(h) / 64          # the weights' sums over rows in 32 bits
        near(grads[2], leaves[2].grad, R * rows * (dy * M * a).sum(0), f"grad_post {W}")
        near(grads[3], leaves[3].grad, R * rows * (gn.double().abs() * um * b * slack).sum(0), f"grad_next {W}")
        if g is None:
            assert grads[4] is None
        else:
            dg = abs(lam) * du * y
            near(grads[4], leaves[4].grad, R * (dg if g.dim() == 2 else dg.sum(1)), "grad_gate " + ("f32" if g.dim() == 1 else D))
    return out, normed, grads


@pytest.mark.parametrize("n,d", [(1, 1), (1, 1024), (2, 7), (3, 32), (5, 257), (7, 1001), (33, 264), (149, 1024), (300, 96), (2, 4096), (3, 8192), (2, 8191),
                                 (5000, 40), (1200, 1024), (3000, 700), (1200, 1300), (700, 2900)])
@pytest.mark.parametrize("kind,gate,weights", [("bf16", "vector", "bf16"), ("f32", "scalar", "f32"), ("bf16", "none", "f32"), ("f32", "vector", "bf16"),
                                               ("bf16", "scalar", "f32")])
def test_sizes(n, d, kind, gate, weights):
    check(make(n + d, n, d, kind, gate, weights), sigmoid=(n + d) % 2 == 0)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("d", [24, 40, 1000, 1024, 2056])
def test_strides_and_alignment(kind, d):
    """Rows further apart, and rows that start on no 16-byte boundary: to the bit what rows side by side give where the way is the same."""
    from paper_2607_07388_b200 import engine
    data = make(3, 37, d, kind, "vector")
    want = check(data, sigmoid=True)

    def spread(x, pad, shift):
        if x is None or x.dim() == 1:
            return None if x is None else x.to(DEV)
        y = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=DEV)
        y[:, shift:shift + x.shape[1]] = x.to(DEV)
        return y[:, shift:shift + x.shape[1]]

    for pad, shift in ((16, 8), (5, 3), (1, 0)):
        got = check(data, sigmoid=True, move=lambda x: spread(x, pad, shift))
        if (pad, shift) == (16, 8) and d % 8 == 0:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            for a, b in zip(got[2], want[2]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_in_place(kind):
    from paper_2607_07388_b200 import engine
    h, m, wp, wn, g, _, _ = (None if x is None else x.to(DEV) for x in make(4, 300, 520, kind, "scalar"))
    out, normed = engine.normed_inject_forward(h, m, wp, wn, g, lam=-2.0)
    version = h._version
    out2, normed2 = engine.normed_inject_forward(h, m, wp, wn, g, lam=-2.0, out=h)
    assert out2 is h and h._version > version and torch.equal(h, out) and torch.equal(normed, normed2)


def test_parts_of_the_gradients():
    from paper_2607_07388_b200 import engine
    data = [None if x is None else x.to(DEV) for x in make(5, 70, 200, "bf16", "vector")]
    full = engine.normed_inject_backward(data[5], data[6], *data[:5])
    for k in range(5):
        want = [i == k for i in range(5)]
        part = engine.normed_inject_backward(data[5], data[6], *data[:5], want=want)
        for i in range(5):
            assert torch.equal(part[i], full[i]) if want[i] else part[i] is None
    # a gradient that does not arrive is one of zeros
    zero = torch.zeros_like(data[5])
    for a, b in zip(engine.normed_inject_backward(None, data[6], *data[:5]), engine.normed_inject_backward(zero, data[6], *data[:5])):
        assert torch.equal(a, b)
    for a, b in zip(engine.normed_inject_backward(data[5], None, *data[:5]), engine.normed_inject_backward(data[5], zero, *data[:5])):
        assert torch.equal(a, b)


def test_no_rows_and_one_row():
    from paper_2607_07388_b200 import engine
    data = [None if x is None else x.to(DEV) for x in make(6, 1, 96, "f32", "scalar")]
    h, m, wp, wn, g, gu, gn = data
    out, normed = engine.normed_inject_forward(h[:0], m[:0], wp, wn, g[:0])
    assert out.shape == normed.shape == (0, 96)
    grads = engine.normed_inject_backward(gu[:0], gn[:0], h[:0], m[:0], wp, wn, g[:0])
    assert grads[0].shape == (0, 96) and not grads[2].any() and not grads[3].any() and grads[4].shape == (0,)


def test_rows_keep_to_themselves():
    """A row's results do not depend on the others, nor on how many there are; NaN in a row stays there; a row of zeros has the norm sqrt(eps)."""
    from paper_2607_07388_b200 import engine
    h, m, wp, wn, g, gu, gn = (x.to(DEV) for x in make(7, 600, 328, "bf16", "vector"))
    out, normed = engine.normed_inject_forward(h, m, wp, wn, g, sigmoid=True)
    for r in (0, 299, 599):
        o, n = engine.normed_inject_forward(h[r:r + 1], m[r:r + 1], wp, wn, g[r:r + 1], sigmoid=True)
        assert torch.equal(o[0], out[r]) and torch.equal(n[0], normed[r])
    bad = m.clone()
    bad[123, 7] = float("nan")
    o, n = engine.normed_inject_forward(h, bad, wp, wn, g, sigmoid=True)
    others = torch.arange(600, device=DEV) != 123
    assert torch.isnan(o[123]).all() and torch.isnan(n[123]).all() and torch.equal(o[others], out[others]) and torch.equal(n[others], normed[others])
    grads = engine.normed_inject_backward(gu, gn, h, bad, wp, wn, g, sigmoid=True)
    clean = engine.normed_inject_backward(gu, gn, h, m, wp, wn, g, sigmoid=True)
    for k in (0, 1, 4):
        assert torch.isnan(grads[k][123]).all() and torch.equal(grads[k][others], clean[k][others])
    z = torch.zeros_like(h[:4])
    o, n = engine.normed_inject_forward(z, z, wp, wn, g[:4], eps=1e-6)
    assert not o.any() and not n.any()


@pytest.mark.parametrize("sigmoid", [False, True])
def test_gates_at_the_ends_of_their_range(sigmoid):
    """A sigmoid of -1000 is 0 and of 1000 is 1, with no gradient; a gate of 0 leaves the row as it is."""
    from paper_2607_07388_b200 import engine
    h, m, wp, wn, _, gu, gn = (None if x is None else x.to(DEV) for x in make(8, 6, 64, "f32", "none"))
    g = torch.tensor([-1000.0, 1000.0, 0.0, -90.0, 90.0, 1.0], device=DEV)
    out, _ = engine.normed_inject_forward(h, m, wp, wn, g, sigmoid=sigmoid)
    grads = engine.normed_inject_backward(gu, gn, h, m, wp, wn, g, sigmoid=sigmoid)
    assert torch.isfinite(out).all() and all(torch.isfinite(x).all() for x in grads)
    if sigmoid:
        assert torch.equal(out[0], h[0]) and not grads[4][:2].any()
    else:
        assert torch.equal(out[2], h[2])


def test_offsets_beyond_32_bits():
    from paper_2607_07388_b200 import engine
    n, d = 2_200_000, 1024
    h = torch.zeros((n, d), dtype=torch.bfloat16, device=DEV)
    m = torch.zeros_like(h)
    tail = make(9, 20, d, "bf16", "none", "f32")
    h[-20:], m[-20:] = tail[0].to(DEV), tail[1].to(DEV)
    wp, wn = tail[2].to(DEV), tail[3].to(DEV)
    out, normed = engine.normed_inject_forward(h, m, wp, wn, lam=0.5)
    o, nn = engine.normed_inject_forward(h[-20:], m[-20:], wp, wn, lam=0.5)
    assert torch.equal(out[-20:], o) and torch.equal(normed[-20:], nn) and not out[:1000].any()
    del normed
    out.zero_()
    out[-20:] = tail[5].to(DEV)
    grads = engine.normed_inject_backward(out, None, h, m, wp, wn, lam=0.5)
    want = engine.normed_inject_backward(tail[5].to(DEV), None, h[-20:], m[-20:], wp, wn, lam=0.5)
    assert torch.equal(grads[0][-20:], want[0]) and torch.equal(grads[1][-20:], want[1])
    assert float((grads[2] - want[2]).abs().max()) <= 2.0 ** -20 * float(want[2].abs().max() + 1) * 20


def test_against_differences():
    """Along a direction e: (f(x + e) - f(x - e)) / 2 in fp32, f the sum of both results weighted by the gradients that arrive.  Second-order
    terms cancel; e is 1e-2 of a unit, so the third is some 1e-6 of f's terms, and fp32 sums of 2 x 40 x 96 terms are off by 1e-6 of theirs."""
    from paper_2607_07388_b200 import engine
    data = [x.to(DEV) for x in make(10, 40, 96, "f32", "vector", zero_row=False)]
    h, m, wp, wn, g, gu, gn = data
    m = m * 10
    kw = dict(sigmoid=True, lam=0.75)
    grads = engine.normed_inject_backward(gu, gn, h, m, wp, wn, g, **kw)
    rng = torch.Generator(device=DEV).manual_seed(1)
    args = [h, m, wp, wn, g]

    def f(a):
        out, normed = engine.normed_inject_forward(*a, **kw)
        return float((out.double() * gu.double()).sum() + (normed.double() * gn.double()).sum())

    for k, grad in enumerate(grads):
        e = torch.randn(args[k].shape, generator=rng, device=DEV) * 1e-2
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + e, args[k] - e
        want = (f(up) - f(down)) / 2
        got = float((grad.double() * e.double()).sum())
        assert abs(got - want) <= 1e-3 * abs(want) + 40 * 96 * 2e-7, (k, got, want)


def test_autograd():
    from paper_2607_07388_b200 import engine
    h, m, wp, wn, g, gu, gn = (x.to(DEV) for x in make(11, 50, 160, "bf16", "scalar"))
    leaves = [x.clone().requires_grad_() for x in (h, m, wp, wn, g)]
    out, normed = engine.normed_inject(*leaves, sigmoid=True, lam=0.3)
    torch.autograd.backward([out, normed], [gu, gn])
    want = engine.normed_inject_backward(gu, gn, h, m, wp, wn, g, sigmoid=True, lam=0.3)
    for x, y in zip(leaves, want):
        assert torch.equal(x.grad, y)
    # one result used, its gradient one number for all elements; only the gate is trained
    g2 = g.clone().requires_grad_()
    _, normed = engine.normed_inject(h, m, wp, wn, g2, sigmoid=True, lam=0.3)
    normed.sum().backward()
    assert torch.equal(g2.grad, engine.normed_inject_backward(None, torch.ones_like(h), h, m, wp, wn, g, sigmoid=True, lam=0.3)[4])


def test_captured_and_two_streams():
    from paper_2607_07388_b200 import engine
    data = [[x.to(DEV) for x in make(s, 700, 512, "bf16", "vector")] for s in (12, 13)]
    want = [(*engine.normed_inject_forward(*d[:5]), *engine.normed_inject_backward(d[5], d[6], *d[:5])) for d in data]
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    got = [[(*engine.normed_inject_forward(*d[:5], stream=s), *engine.normed_inject_backward(d[5], d[6], *d[:5], stream=s)) for _ in range(4)]
           for d, s in zip(data, streams)]
    torch.cuda.synchronize()
    for k in range(2):
        for one in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(one, want[k]))
    held = [x.clone() for x in data[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = (*engine.normed_inject_forward(*held[:5]), *engine.normed_inject_backward(held[5], held[6], *held[:5]))
    for k in (1, 0):
        for a, b in zip(held, data[k]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(made, want[k]))


def test_refusals():
    from paper_2607_07388_b200 import engine
    h, m, wp, wn, g, gu, gn = (x.to(DEV) for x in make(14, 6, 32, "bf16", "vector"))
    for bad in ((h, m.float(), wp, wn, g), (h, m[:5], wp, wn, g), (h.half(), m.half(), wp, wn, g), (h, m, wp[:31], wn, g), (h, m, wp, wn.bfloat16(), g),
                (h, m, wp, wn, g.float()), (h, m, wp, wn, g[:, 0]), (h, m, wp.double(), wn.double(), g), (h.cpu(), m, wp, wn, g), (h.T.contiguous().T, m, wp, wn, g)):
        with pytest.raises(ValueError):
            engine.normed_inject_forward(*bad)
    wide = torch.zeros((2, 8200), device=DEV)
    one = torch.ones(8200, device=DEV)
    from paper_2607_07388_b200.binding import TfeError
    for call in (lambda: engine.normed_inject_forward(wide, wide, one, one), lambda: engine.normed_inject_forward(h, m, wp, wn, g, eps=-1.0),
                 lambda: engine.normed_inject_forward(h, m, wp, wn, g, lam=float("inf")), lambda: engine.normed_inject_forward(h, m, wp, wn, g, out=m),
                 lambda: engine.normed_inject_forward(h, h, wp, wn, g, out=h)):
        with pytest.raises(TfeError):
            call()
    with pytest.raises(ValueError):
        engine.normed_inject_backward(None, None, h, m, wp, wn, g)
    with pytest.raises(ValueError):
        engine.normed_inject_backward(gu.float(), gn, h, m, wp, wn, g)


@pytest.mark.parametrize("seed", range(int(os.environ.get("TFE_RANDOM_CASES", "12"))))
def test_random_sizes(seed):
    rng = random.Random(2000 + seed)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    d = log(1, 8192)
    n = log(1, max(2, 400_000 // d))
    check(make(seed, n, d, rng.choice(["bf16", "f32"]), rng.choice(["none", "scalar", "vector"]), rng.choice(["bf16", "f32"])), sigmoid=rng.random() < 0.5,
          lam=rng.choice([1.0, -0.5, 0.0, 3.0]), eps=rng.choice([1e-6, 1e-5, 1e-2]))
