"""Injection between two norms, forward and gradients, against the formulas in 64 bits."""
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
                                 (5000, 40), (1200, 1024)])
@pytest.mark.parametrize("kind,gate,weights", [("bf16", "vector", "bf16"), ("f32", "scalar", "f32"), ("bf16", "none", "f32"), ("f32", "vector", "bf16"),
                                               ("bf16", "scalar", "f32")])
def test_sizes(n, d, kind, gate, weights):
    check(make(n + d, n, d, kind, gate, weights), sigmoid=(n + d) % 2 == 0)
