"""Softmax cross entropy from hidden states, loss and gradients, against the formulas in 64 bits."""
import math
import os
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
HALF_BF16 = 2.0 ** -8


def reference(h, w, t, g=None):
    """(loss, lse, grad_hidden, grad_weight) in float64; rows without a target, or a gradient, are left out of every sum."""
    h, w, t = h.double(), w.double(), t.long()
    live = (t >= 0) & (t < w.shape[0])
    loss, lse = torch.zeros(len(t), dtype=torch.float64), torch.zeros(len(t), dtype=torch.float64)
    at = live.nonzero()[:, 0]
    z = h[at] @ w.T
    lse[at] = torch.logsumexp(z, 1)
    loss[at] = lse[at] - z.gather(1, t[at][:, None])[:, 0]
    if g is None:
        return loss, lse, None, None
    at = (live & (g != 0)).nonzero()[:, 0]
    p = torch.exp(h[at] @ w.T - lse[at][:, None])
    p[torch.arange(len(at)), t[at]] -= 1
    p *= g[at].double()[:, None]
    gh = torch.zeros_like(h)
    gh[at] = p @ w
    return loss, lse, gh, p.T @ h[at]


def tolerances(h, w, t, g, lse):
    """How far results may be off.  A logit is a sum of d exact products in fp32: each of its d / 16 joined steps off by at most two half
    steps (2^-23) of the sum of magnitudes S.  An exponential adds 2^-22 and three half-steps of its exponent.  G = g p carries
    those, and half a bf16 step of itself; a gradient sums G's errors against the other operand's magnitudes (the worst case: all of
    one sign), and is rounded once.  Sums over the vocabulary and the rows in fp32 add 2^-23 per 16 terms of the magnitudes'."""
    h, w = h.double(), w.double()
    n, d = h.shape
    at = ((t >= 0) & (t < len(w))).nonzero()[:, 0]
    tol_z = torch.zeros(n, dtype=torch.float64)
    size = (h[at].abs() @ w.abs().T)
    tol_z[at] = size.amax(1) * (d / 16 + 2) * 2.0 ** -23
    tol_loss = 2 * tol_z + 2.0 ** -21 + (len(w) / 512 + 64) * 2.0 ** -24 + (lse.abs() + 1) * 2.0 ** -23
    if g is None:
        return tol_loss, None, None
    z = h[at] @ w.T
    p = torch.exp(z - lse[at][:, None])
    ga = g[at].double().abs()[:, None]
    onehot = torch.zeros_like(p)
    onehot[torch.arange(len(at)), t[at].long()] = 1
    rel = (2 * tol_z[at] + 2.0 ** -20 + 4 * 2.0 ** -24 * (z.abs().amax(1) + lse[at].abs()))[:, None]
    G = ga * (p - onehot).abs()
    err = ga * (p + onehot) * rel + G * HALF_BF16
    tol_h = torch.zeros_like(h)
    tol_h[at] = err @ w.abs() + (G @ w.abs()) * (len(w) / 16 + 16) * 2.0 ** -23
    tol_w = err.T @ h[at].abs() + (G.T @ h[at].abs()) * (n / 16 + 16) * 2.0 ** -23
    return tol_loss, tol_h, tol_w


def make(seed, n, v, d, ignored=0.0, know=1.5):
    rng = torch.Generator().manual_seed(seed)
    w = (torch.randn((v, d), generator=rng) * (2.5 / d ** 0.5)).bfloat16()
    t = torch.randint(0, v, (n,), generator=rng)
    h = (torch.randn((n, d), generator=rng) + know * w[t].float()).bfloat16()
    t = torch.where(torch.rand(n, generator=rng) < ignored, torch.randint(0, 2, (n,), generator=rng) * (v + 1) - 1, t).int()
    g = torch.rand(n, generator=rng) + 0.1
    return h, w, t, g


def near(got, want, tol, what):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol + HALF_BF16 * want.abs() * (got.dtype == torch.bfloat16) + 1e-30).all()), (what, float((off - tol).max()), float(off.max()))


def check(h, w, t, g, run=None):
    from paper_2607_07388_b200 import engine
    hd, wd, td, gd = (x.to(DEV) for x in (h, w, t, g))
    if run is None:
        loss, lse = engine.xent_forward(hd, wd, td)
        gh, gw = engine.xent_backward(gd, hd, wd, td, lse)
    else:
        loss, lse, gh, gw = run(hd, wd, td, gd)
    e_loss, e_lse, e_gh, e_gw = reference(h, w, t, g)
    tol, tol_h, tol_w = tolerances(h, w, t, g, e_lse)
    near(loss, e_loss, tol, "loss")
    near(lse, e_lse, tol, "lse")
    near(gh, e_gh, tol_h, "grad_hidden")
    near(gw, e_gw, tol_w, "grad_weight")
    away = (t < 0) | (t >= len(w))
    assert not loss.cpu()[away].any() and not lse.cpu()[away].any() and not gh.cpu()[away].any()
    assert engine.xent_status() == 0
    return loss, lse, gh, gw


@pytest.mark.parametrize("n,v,d", [(1, 1, 8), (1, 300, 64), (2, 17, 72), (7, 255, 136), (31, 257, 256), (33, 512, 264), (128, 1000, 128),
                                   (129, 1001, 320), (255, 770, 512), (257, 2049, 40), (300, 5000, 1024), (513, 129, 1000), (1000, 300, 64),
                                   (64, 20_003, 256), (700, 9000, 520)])
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_sizes(n, v, d, ignored):
    check(*make(n + v + d, n, v, d, ignored))


def rel(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("n", [15, 16, 17, 32, 48, 63, 64, 65, 66, 256])
def test_row_counts_at_which_the_way_changes(n):
    h, w, t, g = make(n, n, 1031, 192, 0.1)
    loss, lse, gh, gw = check(h, w, t, g)
    _, _, e_gh, e_gw = reference(h, w, t, g)
    # both roundings of a gradient, each 2^-8 at most of what is rounded: of the result, and of G, whose errors have random signs
    assert rel(gh, e_gh) <= 2.0 ** -7 and rel(gw, e_gw) <= 2.0 ** -7


@pytest.mark.parametrize("n", [5, 40, 200, 300])
def test_rows_without_a_target(n):
    """Whatever an ignored row holds, and in whatever number: no result but its own zeros depends on it."""
    from paper_2607_07388_b200 import engine
    h, w, t, g = make(7, n, 777, 128)
    t[::3] = torch.tensor([-1, 777, 2 ** 31 - 1, -2 ** 31] * n, dtype=torch.int32)[:len(t[::3])]
    ok = check(h, w, t, g)
    h2 = h.clone()
    h2[::3] = float("nan")
    h2[0, 0] = float("inf")
    again = [x.cpu() for x in engine.xent_forward(*(x.to(DEV) for x in (h2, w, t)))]
    assert torch.equal(again[0], ok[0].cpu()) and torch.equal(again[1], ok[1].cpu())
    gh, gw = engine.xent_backward(g.to(DEV), h2.to(DEV), w.to(DEV), t.to(DEV), ok[1])
    assert torch.equal(gh, ok[2]) and torch.equal(gw, ok[3])
    # a gradient of zero takes its row out just so
    g2 = g.clone()
    t2 = torch.where(t < 0, 5, t).int()
    t2[t2 >= 777] = 5
    g2[::3] = 0.0
    gh, gw = engine.xent_backward(g2.to(DEV), h2.to(DEV), w.to(DEV), t2.to(DEV), ok[1])
    assert torch.equal(gh, ok[2]) and torch.equal(gw, ok[3])
    # no row at all
    none = torch.full_like(t, -1)
    loss, lse, gh, gw = check(h, w, none, g, run=lambda a, b, c, d: (*engine.xent_forward(a, b, c), *engine.xent_backward(d, a, b, c, torch.zeros(n, device=DEV))))
    assert not gh.any() and not gw.any() and not loss.any()


def test_no_rows():
    from paper_2607_07388_b200 import engine
    w = torch.randn(100, 64, device=DEV).bfloat16()
    h, t = w[:0], torch.empty(0, dtype=torch.int32, device=DEV)
    loss, lse = engine.xent_forward(h, w, t)
    gh, gw = engine.xent_backward(loss, h, w, t, lse)
    assert loss.shape == lse.shape == (0,) and gh.shape == (0, 64) and gw.shape == (100, 64) and not gw.any()
    assert engine.xent_backward(loss, h, w, t, lse, want_weight=False)[1] is None


@pytest.mark.parametrize("n", [9, 150, 700])
def test_values_that_are_not_finite_stay_where_they_belong(n):
    from paper_2607_07388_b200 import engine
    h, w, t, g = make(8, n, 500, 64)
    clean = [x.cpu() for x in engine.xent_forward(*(x.to(DEV) for x in (h, w, t)))]
    bad = h.clone()
    bad[n // 2, 3] = float("nan")
    loss, lse = engine.xent_forward(*(x.to(DEV) for x in (bad, w, t)))
    others = torch.arange(n) != n // 2
    assert torch.isnan(loss[n // 2]) and torch.isnan(lse[n // 2])
    assert torch.equal(loss.cpu()[others], clean[0][others]) and torch.equal(lse.cpu()[others], clean[1][others])
    gh, gw = engine.xent_backward(g.to(DEV), bad.to(DEV), w.to(DEV), t.to(DEV), lse)
    assert torch.isnan(gh[n // 2]).all() and torch.isfinite(gh.cpu()[others].float()).all() and torch.isnan(gw).any()
    # a weight of -inf against hidden states above 0: a token that cannot come, whose row of grad_weight is zeros.  (0 times -inf reaches
    # grad_hidden, as it does in the formula.)
    h0 = h.clone()
    h0[:, 5] = 0.5
    w0 = w.clone()
    w0[77, 5] = -float("inf")
    t0 = torch.where(t == 77, 78, t).int()
    loss, lse = engine.xent_forward(*(x.to(DEV) for x in (h0, w0, t0)))
    _, gw = engine.xent_backward(g.to(DEV), h0.to(DEV), w0.to(DEV), t0.to(DEV), lse, want_hidden=False)
    keep = torch.arange(500) != 77
    assert not gw[77].any() and torch.isfinite(gw.float()).all()
    e_loss = reference(h0, w0[keep], torch.where(t0 > 77, t0 - 1, t0))[0]
    assert float((loss.double().cpu() - e_loss).abs().max()) <= 1e-5 * float(e_loss.abs().max() + 1)
    # a logit of +inf: NaN
    bad = h.clone()
    bad[1] = 0
    bad[1, 0] = float("inf")
    loss, _ = engine.xent_forward(*(x.to(DEV) for x in (bad, w, t)))
    assert torch.isnan(loss[1])


@pytest.mark.parametrize("n", [40, 400])
def test_one_target_for_many_rows(n):
    """More rows of one target than are corrected one by one, next to targets of few rows."""
    h, w, t, g = make(9, n, 300, 256)
    t[:n // 2] = 31
    t[n // 2:n // 2 + 6] = 32
    t[n // 2 + 6:n // 2 + 8] = 299
    loss, lse, gh, gw = check(h, w, t, g)
    _, _, e_gh, e_gw = reference(h, w, t, g)
    assert rel(gw[31:33], e_gw[31:33]) <= 2.0 ** -7 and rel(gw[299], e_gw[299]) <= 2.0 ** -7


def test_targets_of_one_row_are_exact():
    """Weights that matter little but for the target: the gradients are their own rounding and hardly more, since G's rounding at the target is
    made up for.  G elsewhere is below 1 / 4,000 of it, so its rounding adds at most sqrt(4,000) / 4,000 of 2^-8 in the 2-norm."""
    h, w, t, g = make(10, 24, 4000, 512, know=0.0)
    w = (w.float() * 0.01).bfloat16()
    t = (torch.arange(24) * 161 + 5).int()
    _, _, gh, gw = check(h, w, t, g)
    _, _, e_gh, e_gw = reference(h, w, t, g)
    for r in range(24):
        assert rel(gw[t[r]], e_gw[t[r]]) <= 2.0 ** -8 * 1.05
    assert bool(((gw.double().cpu() - e_gw)[t.long()].abs() <= e_gw[t.long()].abs() * 2.0 ** -8 * 1.02 + e_gw.abs().max() * 2.0 ** -12).all())


@pytest.mark.parametrize("n", [30, 130, 600])
def test_large_and_small_losses(n):
    """Logits of hundreds, and rows that are sure of their target: the loss near zero is exp(-gap), not a difference of rounded numbers
    beyond what the logits' own sum is off by."""
    h, w, t, g = make(11, n, 900, 64, know=0.0)
    sharp = (h.float() * 0.3 + 6 * w[t.long()].float()).bfloat16()
    check(sharp, w, t, g)
    check((h.float() * 100).bfloat16(), w, t, g)


@pytest.mark.parametrize("n", [20, 300])
def test_rows_further_apart(n):
    from paper_2607_07388_b200 import engine
    h, w, t, g = make(12, n, 450, 136)
    hb, wb = torch.full((n, 200), float("nan"), device=DEV).bfloat16(), torch.full((450, 144), float("nan"), device=DEV).bfloat16()
    hb[:, 16:152] = h.to(DEV)
    wb[:, 8:] = w.to(DEV)
    want = check(h, w, t, g)
    got = check(h, w, t, g, run=lambda a, b, c, d: (lambda f: (*f, *engine.xent_backward(d, hb[:, 16:152], wb[:, 8:], c, f[1])))(engine.xent_forward(hb[:, 16:152], wb[:, 8:], c)))
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_one_gradient_alone():
    from paper_2607_07388_b200 import engine
    h, w, t, g = (x.to(DEV) for x in make(13, 300, 600, 128))
    loss, lse = engine.xent_forward(h, w, t)
    gh, gw = engine.xent_backward(g, h, w, t, lse)
    a, none = engine.xent_backward(g, h, w, t, lse, want_weight=False)
    assert none is None and torch.equal(a, gh)
    none, b = engine.xent_backward(g, h, w, t, lse, want_hidden=False)
    assert none is None and torch.equal(b, gw)


def test_several_pieces_of_the_vocabulary():
    """4,096 rows x 70,001: G takes three pieces, the last one short.  The reference runs on the GPU in 64 bits; 2-norms."""
    from paper_2607_07388_b200 import engine
    n, v, d = 4096, 70_001, 64
    rng = torch.Generator(device=DEV).manual_seed(14)
    w = (torch.randn((v, d), generator=rng, device=DEV) * 0.3).bfloat16()
    t = torch.randint(0, v, (n,), generator=rng, device=DEV).int()
    h = (torch.randn((n, d), generator=rng, device=DEV) + w[t.long()].float()).bfloat16()
    g = torch.rand(n, generator=rng, device=DEV)
    t[5::7] = -1
    loss, lse = engine.xent_forward(h, w, t)
    gh, gw = engine.xent_backward(g, h, w, t, lse)
    live = t >= 0
    z = h.double()[live] @ w.double().T
    e_lse = torch.logsumexp(z, 1)
    assert float((lse[live].double() - e_lse).abs().max()) <= 4e-5          # of 14: 3e-6 as a fraction
    z.sub_(e_lse[:, None]).exp_()
    z[torch.arange(len(z)), t[live].long()] -= 1
    z *= g[live].double()[:, None]
    e_gh, e_gw = torch.zeros_like(h, dtype=torch.float64), z.T @ h.double()[live]
    e_gh[live] = z @ w.double()
    assert float((gh.double() - e_gh).norm() / e_gh.norm()) <= 2.0 ** -8 and float((gw.double() - e_gw).norm() / e_gw.norm()) <= 2.0 ** -8
    assert float((gw.double() - e_gw)[-300:].norm() / e_gw[-300:].norm()) <= 2.0 ** -7
    # the same again: to the bit
    gh2, gw2 = engine.xent_backward(g, h, w, t, lse)
    assert torch.equal(gh, gh2) and torch.equal(gw, gw2)


def test_offsets_beyond_32_bits():
    """A projection of 2.2 billion elements: the last rows' results are those of a small projection made of them."""
    from paper_2607_07388_b200 import engine
    v, d, n = 4_200_000, 520, 5
    rng = torch.Generator(device=DEV).manual_seed(15)
    w = torch.zeros((v, d), dtype=torch.bfloat16, device=DEV)
    tail = torch.randn((64, d), generator=rng, device=DEV).bfloat16()
    w[-64:] = tail
    h = torch.randn((n, d), generator=rng, device=DEV).bfloat16()
    t = torch.tensor([v - 1, v - 64, v - 30, 7, -1], dtype=torch.int32, device=DEV)
    g = torch.ones(n, device=DEV)
    loss, lse = engine.xent_forward(h, w, t)
    z = h.double() @ tail.double().T
    e_lse = torch.log(torch.exp(z).sum(1) + (v - 64))
    e_loss = e_lse - torch.stack([z[0, 63], z[1, 0], z[2, 34], z[3, 0] * 0, z[4, 0]])
    assert float((loss[:4].double() - e_loss[:4]).abs().max()) <= 1e-4 and float(loss[4]) == 0.0
    gh, gw = engine.xent_backward(g, h, w, t, lse)
    p = torch.exp(z - e_lse[:, None])
    for r, c in ((0, 63), (1, 0), (2, 34)):
        p[r, c] -= 1
    p[4] = 0
    e_gw = p.T @ h.double()
    assert float((gw[-64:].double() - e_gw).norm() / e_gw.norm()) <= 2.0 ** -7
    assert float((gh[:4].double() - (p @ tail.double())[:4]).norm() / (p @ tail.double())[:4].norm()) <= 2.0 ** -7
    assert engine.xent_status() == 0


def test_gradients_against_differences():
    """The loss at h + e and h - e, where h, e and both sums are bf16 numbers without rounding: half their difference is the gradient along
    e up to the third derivative.  With |z(e)| <= 0.1 that is at most 0.1^3 / 6 per unit of g; the losses' own error is 1e-5."""
    from paper_2607_07388_b200 import engine
    rng = torch.Generator().manual_seed(16)
    n, v, d = 90, 400, 64
    h = (torch.randint(-32, 33, (n, d), generator=rng) / 16.0).bfloat16()
    w = (torch.randint(-32, 33, (v, d), generator=rng) / 64.0).bfloat16()
    t, g = torch.randint(0, v, (n,), generator=rng).int(), torch.rand(n, generator=rng) + 0.5
    hd, wd, td, gd = (x.to(DEV) for x in (h, w, t, g))
    _, lse = engine.xent_forward(hd, wd, td)
    gh, gw = engine.xent_backward(gd, hd, wd, td, lse)
    for k in range(4):
        e = (torch.randint(-1, 2, (n, d), generator=rng) / 64.0).bfloat16()
        up, down = (engine.xent_forward((h.float() + s * e.float()).bfloat16().to(DEV), wd, td)[0].double().cpu() for s in (1, -1))
        want = float((g * (up - down) / 2).sum())
        got = float((gh.double().cpu() * e.double()).sum())
        # each row: third derivative, losses, and the gradient's roundings against e
        slack = n * 1.5 * (0.1 ** 3 / 6 + 1e-5) + float((gh.double().cpu().abs() * e.double().abs()).sum()) * 2.0 ** -7
        assert abs(got - want) <= slack and abs(want) > 1e-3
        e = (torch.randint(-1, 2, (v, d), generator=rng) / 256.0).bfloat16()
        up, down = (engine.xent_forward(hd, (w.float() + s * e.float()).bfloat16().to(DEV), td)[0].double().cpu() for s in (1, -1))
        want = float((g * (up - down) / 2).sum())
        got = float((gw.double().cpu() * e.double()).sum())
        slack = n * 1.5 * (0.1 ** 3 / 6 + 1e-5) + float((gw.double().cpu().abs() * e.double().abs()).sum()) * 2.0 ** -7
        assert abs(got - want) <= slack


def test_autograd():
    from paper_2607_07388_b200 import engine
    h, w, t, g = make(17, 270, 1300, 64, 0.2)
    hd, wd, td = h.to(DEV).requires_grad_(), w.to(DEV).requires_grad_(), t.to(DEV)
    loss = engine.linear_cross_entropy(hd, wd, td)
    (loss * g.to(DEV)).sum().backward()
    _, _, e_gh, e_gw = reference(h, w, t, g)
    _, tol_h, tol_w = tolerances(h, w, t, g, reference(h, w, t)[1])
    near(hd.grad, e_gh, tol_h, "grad_hidden")
    near(wd.grad, e_gw, tol_w, "grad_weight")
    # a mean, whose gradient is one number for all rows; one leaf only
    hd.grad = None
    engine.linear_cross_entropy(hd, wd.detach(), td).sum().backward()
    gh, none = engine.xent_backward(torch.ones(270, device=DEV), hd.detach(), wd.detach(), td, engine.xent_forward(hd.detach(), wd.detach(), td)[1], want_weight=False)
    assert none is None and torch.equal(hd.grad, gh)


@pytest.mark.parametrize("n", [20, 100, 400])
def test_captured_and_replayed(n):
    from paper_2607_07388_b200 import engine
    data = [tuple(x.to(DEV) for x in make(s, n, 2100, 72, 0.3)) for s in (18, 19)]
    want = []
    for h, w, t, g in data:
        f = engine.xent_forward(h, w, t)
        want.append((*f, *engine.xent_backward(g, h, w, t, f[1])))
    h, w, t, g = (x.clone() for x in data[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        engine.xent_backward(g, h, w, t, engine.xent_forward(h, w, t)[1])
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    results = []
    for graph in graphs:                    # two graphs over the same inputs
        with torch.cuda.graph(graph):
            f = engine.xent_forward(h, w, t)
            results.append((*f, *engine.xent_backward(g, h, w, t, f[1])))
    for k in (1, 0, 1):
        for x, y in zip((h, w, t, g), data[k]):
            x.copy_(y)
        for graph, got in zip(graphs, results):
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(got, want[k]):
                assert torch.equal(a, b)
    assert engine.xent_status() == 0


def test_two_streams_at_once():
    from paper_2607_07388_b200 import engine
    data = [tuple(x.to(DEV) for x in make(s, 500, 3000, 128, 0.1)) for s in (20, 21)]
    want = []
    for h, w, t, g in data:
        f = engine.xent_forward(h, w, t)
        want.append((*f, *engine.xent_backward(g, h, w, t, f[1])))
    streams = [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, (h, w, t, g) in enumerate(data):
            f = engine.xent_forward(h, w, t, stream=streams[k])
            got[k].append((*f, *engine.xent_backward(g, h, w, t, f[1], stream=streams[k])))
    torch.cuda.synchronize()
    for k in range(2):
        for one in got[k]:
            for a, b in zip(one, want[k]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("n", [10, 100, 400])
def test_a_wait_that_runs_out(n):
    """Every wait counts as run out from the start: NaN in what has a target, a report once, and all well afterwards."""
    from paper_2607_07388_b200 import binding as tfe, engine
    h, w, t, g = (x.to(DEV) for x in make(22, n, 900, 64, 0.2))
    loss, lse = engine.xent_forward(h, w, t)
    gh, gw = engine.xent_backward(g, h, w, t, lse)
    assert engine.xent_status() == 0
    tfe.tfe_xent_give_up(True)
    try:
        bad, _ = engine.xent_forward(h, w, t)
        assert engine.xent_status() != 0 and engine.xent_status() == 0
        bh, bw = engine.xent_backward(g, h, w, t, lse)
        assert engine.xent_status() != 0 and engine.xent_status() == 0
    finally:
        tfe.tfe_xent_give_up(False)
    live = (t >= 0) & (t < 900)
    assert torch.isnan(bad[live]).all() and not bad[~live].any() and torch.isnan(bh[live]).all() and torch.isnan(bw).all()
    again = engine.xent_forward(h, w, t)
    assert torch.equal(again[0], loss) and torch.equal(engine.xent_backward(g, h, w, t, lse)[1], gw) and engine.xent_status() == 0


def test_refusals():
    from paper_2607_07388_b200 import engine
    h, w, t, g = (x.to(DEV) for x in make(23, 8, 40, 64))
    lse = torch.zeros(8, device=DEV)
    for bad in ((h.float(), w, t), (h, w.float(), t), (h, w, t.long()), (h, w[:, :56], t), (h[:, :60], w[:, :60], t), (h[:, 1:57], w[:, :56], t), (h.cpu(), w, t),
                (h, w, t[:7]), (h.T.contiguous().T, w, t), (h, w[:0], t), (h[0], w, t), (h, w, t.cpu())):
        with pytest.raises(ValueError):
            engine.xent_forward(*bad)
    for kw in (dict(grad_loss=g.double()), dict(lse=lse[:4]), dict(grad_loss=g.expand(2, 8)), dict(target=t.long())):
        a = dict(grad_loss=g, hidden=h, weight=w, target=t, lse=lse) | kw
        with pytest.raises(ValueError):
            engine.xent_backward(**a)
    assert engine.xent_backward(g, h, w, t, lse, want_hidden=False, want_weight=False) == (None, None)


@pytest.mark.parametrize("seed", range(int(os.environ.get("TFE_RANDOM_CASES", "12"))))
def test_random_sizes(seed):
    rng = random.Random(1000 + seed)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n, d = log(1, 4000), 8 * log(1, 90)
    v = log(1, max(2, min(6000, 500_000_000 // (n * d))))
    h, w, t, g = make(seed, n, v, d, rng.choice([0.0, 0.0, 0.3, 0.9]), rng.choice([0.0, 1.5, 4.0]))
    pick = torch.Generator().manual_seed(seed)
    if rng.random() < 0.3:              # one id for half of the rows
        t = torch.where(torch.rand(n, generator=pick) < 0.5, torch.full_like(t, rng.randrange(v)), t)
    if rng.random() < 0.3:              # gradients of either sign, and none
        g = torch.where(torch.rand(n, generator=pick) < 0.4, 0.0, g - 0.6)
    check(h, w, t, g)


@pytest.mark.parametrize("n,v,d", [(70, 300, 65_536), (300, 700, 40_008), (70_000, 500, 64), (33_000, 3000, 128), (5, 1_000_000, 64), (300, 1_000_000, 64)])
def test_long_sides(n, v, d):
    """The widest rows, many rows, a large vocabulary; the reference runs on the GPU in 64 bits, 2-norms.  A gradient carries its own rounding and
    what is left of G's, 2^-8 at most each and of random signs: 2^-8 together.  A loss of some units carries logits that are sums of parts of
    512 k, each part off by at most 32 steps of 2^-23 of its size and those parts' sum by d / 512 half-steps: 5e-6."""
    from paper_2607_07388_b200 import engine
    rng = torch.Generator(device=DEV).manual_seed(n + v + d)
    w = (torch.randn((v, d), generator=rng, device=DEV) * (2.5 / d ** 0.5)).bfloat16()
    t = torch.randint(0, v, (n,), generator=rng, device=DEV).int()
    h = (torch.randn((n, d), generator=rng, device=DEV) + w[t.long()].float()).bfloat16()
    t[torch.rand(n, generator=rng, device=DEV) < 0.2] = -1
    g = torch.rand(n, generator=rng, device=DEV) - 0.3
    loss, lse = engine.xent_forward(h, w, t)
    gh, gw = engine.xent_backward(g, h, w, t, lse)
    e_loss, e_gh, e_gw = (torch.zeros(s, dtype=torch.float64, device=DEV) for s in ((n,), (n, d), (v, d)))
    for rows in (t >= 0).nonzero()[:, 0].split(max(1, (1 << 26) // v)):
        z, at = h[rows].double() @ w.double().T, t[rows].long()
        k, norm = torch.arange(len(rows), device=DEV), torch.logsumexp(z, 1)
        e_loss[rows] = norm - z[k, at]
        p = z.sub_(norm[:, None]).exp_()
        p[k, at] -= 1
        p *= g[rows].double()[:, None]
        e_gh[rows] = p @ w.double()
        e_gw += p.T @ h[rows].double()
    for got, want, most in ((loss, e_loss, 5e-6), (gh, e_gh, 2.0 ** -8), (gw, e_gw, 2.0 ** -8)):
        assert float((got.double() - want).norm() / want.norm()) <= most
    assert engine.xent_status() == 0
