"""Softmax cross entropy from hidden states, loss and gradients, against the formulas in 64 bits."""
import numpy as np
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
