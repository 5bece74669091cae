"""Injection between norms and clipping at the ends of what their arguments allow."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def formula(h, m, wp, wn, gate, sigmoid, lam, eps):
    s = gate[:, None] if gate.dim() == 1 else gate
    s = torch.sigmoid(s) if sigmoid else s
    u = h + lam * s * (wp * m / torch.sqrt((m * m).mean(1, keepdim=True) + eps))
    return u, wn * u / torch.sqrt((u * u).mean(1, keepdim=True) + eps)


def both(data, **kw):
    """(gradients of the call, of the formula in float64)"""
    from paper_2607_07388_b200 import engine
    h, m, wp, wn, gate, gu, gn = data
    got = engine.normed_inject_backward(gu.to(DEV), gn.to(DEV), *(x.to(DEV) for x in (h, m, wp, wn, gate)), **kw)
    leaves = [x.double().requires_grad_() for x in (h, m, wp, wn, gate)]
    torch.autograd.backward(list(formula(*leaves, **kw)), [gu.double(), gn.double()])
    return [x.double().cpu() for x in got], [x.grad for x in leaves]


def make(seed, n, d, kind, gate):
    rng = torch.Generator().manual_seed(seed)
    h, m, gu, gn = (torch.randn((n, d), generator=rng).to(TYPES[kind]) for _ in range(4))
    wp, wn = (1 + 0.3 * torch.randn(d, generator=rng) for _ in range(2))
    g = torch.randn(n, generator=rng) if gate == "scalar" else torch.randn((n, d), generator=rng).to(TYPES[kind])
    return h, m, wp, wn, g, gu, gn


@pytest.mark.parametrize("kind,gate", [("f32", "scalar"), ("f32", "vector"), ("bf16", "scalar"), ("bf16", "vector")])
@pytest.mark.parametrize("d", [64, 1001, 2048])
def test_gates_that_are_open_or_shut(kind, gate, d):
    """The derivative of a sigmoid far from 0 as a fraction of itself.  As elsewhere every term of a result is off by at most 2^-18 of its magnitude,
    and as much again for the exponential: 2^-22, and half-steps of an exponent of up to 29."""
    data = list(make(1, 18, d, kind, gate))
    x = torch.tensor([8.0, -8.0, 12.0, -12.0, 15.0, -15.0, 17.0, -17.0, 20.0])
    data[4] = (x.repeat(2) if gate == "scalar" else x.repeat(2 * d).view(2 * d, 9).T.reshape(18, d).to(TYPES[kind])).contiguous()
    got, want = both(data, sigmoid=True, lam=0.75, eps=1e-6)
    h, m, wp, wn, g, gu, gn = (t.double() for t in data)
    s = torch.sigmoid(g if g.dim() == 2 else g[:, None])
    slope = s * torch.sigmoid(-(g if g.dim() == 2 else g[:, None]))
    y = wp.abs() * m.abs() / torch.sqrt((m * m).mean(1, keepdim=True) + 1e-6)
    um = h.abs() + 0.75 * s * y
    u = formula(h, m, wp, wn, g, True, 0.75, 1e-6)[0]
    b = 1 / torch.sqrt((u * u).mean(1, keepdim=True) + 1e-6)
    t = (wn * gn).abs()
    du = (gu.abs() + b * t + um * b ** 3 * (um * t).mean(1, keepdim=True)) * (1 + (um * um).mean(1, keepdim=True) * b * b)
    tol = 2.0 ** -17 * 0.75 * du * y * slope
    tol = tol if g.dim() == 2 else tol.sum(1)
    off = (got[4] - want[4]).abs()
    own = HALF[torch.float32 if gate == "scalar" else TYPES[kind]]
    assert bool((off <= tol + own * (want[4].abs() + tol)).all()), float((off / want[4].abs()).max())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [1e-30, 1e-37])
def test_rows_of_zeros_with_a_small_eps(kind, eps):
    """Padding: h and m are zeros, both norms are sqrt(eps), and the gradient is what arrives divided by it."""
    data = make(2, 40, 200, kind, "scalar")
    for x in data[:2]:
        x[::3] = 0
    if eps < 1e-30:
        data[6].mul_(2.0 ** -20)         # (what arrives at a norm leaves it times 1 / sqrt(eps), and times that again at m)
        data[5].mul_(2.0 ** -20)
    got, want = both(data, sigmoid=False, lam=0.75, eps=eps)
    for i, (a, e) in enumerate(zip(got, want)):
        assert bool(torch.isfinite(a).all()), i
    zeros = torch.arange(40) % 3 == 0
    for i in (0, 1):
        own = HALF[TYPES[kind]]
        assert bool(((got[i][zeros] - want[i][zeros]).abs() <= (2.0 ** -18 + own) * want[i][zeros].abs()).all()), i


@pytest.mark.parametrize("scale", [-18, -19])
def test_rows_near_the_end_of_the_range(scale):
    """Rows whose mean squares are near 1e-38, without eps: the norm's gradient is of the size of what arrives, over the row's."""
    data = [x.clone() for x in make(3, 20, 96, "f32", "scalar")]
    data[0] *= 10.0 ** scale * 3
    data[1] *= 10.0 ** scale * 3
    data[4] *= 10.0 ** scale
    data[5] *= 0.0
    got, want = both(data, sigmoid=False, lam=1.0, eps=0.0)
    for i in (0, 3):
        assert bool(torch.isfinite(got[i]).all()), i
        # the two parts of a norm's gradient are of one size: taken by the row's largest element
        most = want[i].abs().amax(-1, keepdim=True)
        assert bool(((got[i] - want[i]).abs() <= 2.0 ** -15 * most).all()), (i, float(((got[i] - want[i]).abs() / most).max()))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1.0, 1e-5, 1e-6])
def test_clipping_by_a_factor_below_the_normal_numbers(kind, max_norm):
    """max_norm / norm below 2^-126: the results are ordinary numbers, off by the factor's rounding and their own."""
    from paper_2607_07388_b200 import engine
    rng = torch.Generator().manual_seed(4)
    x = [(torch.randn(n, generator=rng) * 3e36).to(TYPES[kind]) for n in (1000, 7, 2000)]
    norm = float(torch.cat([t.double() for t in x]).norm())
    assert norm < 3e38
    for out in (None, [torch.empty_like(t, device=DEV) for t in x]):
        a = [t.to(DEV) for t in x]
        got = engine.clip_grad_norm(a, max_norm, out=out)
        assert abs(float(got) - norm) <= 2.0 ** -22 * norm
        for t, r in zip(x, out or a):
            want = t.double() * (max_norm / norm)
            assert bool(((r.double().cpu() - want).abs() <= (2.0 ** -23 + HALF[TYPES[kind]]) * want.abs() + 2.0 ** -149).all())
