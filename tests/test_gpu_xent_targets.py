"""Softmax cross entropy where the target decides: logits of -inf, rows that are sure of their target, ids of many rows."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
HALF_BF16 = 2.0 ** -8


def half_step(x):
    """Half the distance between bf16 numbers at x: no rounding is off by more."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -126))) - 8)


def exact(h, w, t, g):
    """(loss, lse, G, grad_hidden, grad_weight) in float64, G at the target as minus the sum of the others: nothing cancels.  Every row has a target."""
    h, w, t = h.double(), w.double(), t.long()
    rows = torch.arange(len(t))
    z = h @ w.T
    zt = z[rows, t].clone()
    z[rows, t] = -float("inf")
    others = torch.logsumexp(z, 1)
    x = others - zt
    loss = torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))
    lse = torch.maximum(others, zt) + torch.log1p(torch.exp(-x.abs()))
    G = torch.exp(z - lse[:, None])
    G[rows, t] = -G.sum(1)
    G *= g.double()[:, None]
    return loss, lse, G, G @ w, G.T @ h


def logit_error(h, w):
    """A logit is a sum of d exact products in fp32: each of its d / 16 joined steps off by at most two half steps (2^-23) of the sum of magnitudes."""
    return (h.double().abs() @ w.double().abs().T).amax(1) * (h.shape[1] / 16 + 2) * 2.0 ** -23


def relative(h, w, lse):
    """How far a probability, or a sum of them, may be off as a fraction: the errors of two logits, an exponential (2^-22) with four half-steps
    of its exponent, and a sum over the vocabulary."""
    return 2 * logit_error(h, w) + 2.0 ** -20 + 4 * 2.0 ** -24 * (2 * lse.abs() + 40) + (len(w) / 512 + 64) * 2.0 ** -24


def check_loss(h, w, t):
    """The loss as a fraction of itself, however near zero."""
    from paper_2607_07388_b200 import engine
    loss, lse = engine.xent_forward(*(x.to(DEV) for x in (h, w, t)))
    e_loss, e_lse, *_ = exact(h, w, t, torch.ones(len(t)))
    rel = relative(h, w, e_lse)
    off = (loss.double().cpu() - e_loss).abs()
    assert bool((off <= e_loss * (rel + 2.0 ** -23)).all()), ("loss", float((off / e_loss).max()))
    assert bool(((lse.double().cpu() - e_lse).abs() <= rel + 2.0 ** -23 * e_lse.abs()).all())
    assert engine.xent_status() == 0
    return loss, lse


def check(h, w, t, g):
    """Loss and gradients: everything as a fraction of what it is a sum of.  G's entries are rounded to bf16 but for the targets', whose rounding
    is made up for; sums in fp32 add 2^-23 per 16 terms; results are rounded once."""
    from paper_2607_07388_b200 import engine
    loss, lse = check_loss(h, w, t)
    hd, wd, td, gd = (x.to(DEV) for x in (h, w, t, g))
    gh, gw = engine.xent_backward(gd, hd, wd, td, lse)
    _, e_lse, G, e_gh, e_gw = exact(h, w, t, g)
    n, (v, d) = len(t), w.shape
    rel = relative(h, w, e_lse)
    onehot = torch.zeros_like(G)
    onehot[torch.arange(n), t.long()] = 1
    err = G.abs() * (rel[:, None] + HALF_BF16 * (1 - onehot))
    A, B = w.double().abs(), h.double().abs()
    tol_h = err @ A + (G.abs() @ A) * (v / 16 + 16) * 2.0 ** -23
    tol_w = err.T @ B + (G.abs().T @ B) * (n / 16 + 16) * 2.0 ** -23
    for got, want, tol, what in ((gh, e_gh, tol_h, "grad_hidden"), (gw, e_gw, tol_w, "grad_weight")):
        off = (got.double().cpu() - want).abs()
        allowed = tol + half_step(want.abs() + tol)
        assert bool((off <= allowed).all()), (what, float((off / allowed).max()), float((off - allowed).max()))
    assert engine.xent_status() == 0
    return loss, lse, gh, gw


def weights(rng, v, d):
    return (torch.randn((v, d), generator=rng) * (2.5 / d ** 0.5)).bfloat16()


@pytest.mark.parametrize("n", [9, 150, 700])
def test_a_target_that_cannot_come(n):
    """A weight of -inf: the id's logit is -inf in every row.  A row that has it as its target has a loss of +inf and a finite log-sum-exp, and
    its gradient is finite but where it meets that weight itself."""
    from paper_2607_07388_b200 import engine
    rng = torch.Generator().manual_seed(n)
    w = weights(rng, 500, 64)
    t = torch.randint(0, 500, (n,), generator=rng)
    h = (torch.randn((n, 64), generator=rng) + 1.5 * w[t].float()).bfloat16()
    t = torch.where(t == 77, 78, t).int()
    g = torch.rand(n, generator=rng) + 0.1
    h[:, 5] = 0.5
    w[77, 5] = -float("inf")
    r = n // 2
    t[r] = 77
    loss, lse = engine.xent_forward(*(x.to(DEV) for x in (h, w, t)))
    keep = torch.arange(500) != 77
    z = h.double() @ w[keep].double().T
    e_lse = torch.logsumexp(z, 1)
    assert float((lse.double().cpu() - e_lse).abs().max()) <= 1e-5 * float(e_lse.abs().max() + 1)
    rest = torch.arange(n) != r
    assert float(loss[r]) == float("inf") and bool(torch.isfinite(loss.cpu()[rest]).all())
    gh, gw = engine.xent_backward(*(x.to(DEV) for x in (g, h, w, t)), lse)
    G = torch.zeros((n, 500), dtype=torch.float64)
    G[:, keep] = torch.exp(z - e_lse[:, None])
    G[torch.arange(n), t.long()] -= 1
    G *= g.double()[:, None]
    e_gw = G.T @ h.double()
    assert bool(torch.isfinite(gw.float()).all())
    # both roundings, of G and of the result, are 2^-8 at most of what is rounded
    assert float((gw.double().cpu() - e_gw).norm() / e_gw.norm()) <= 2.0 ** -7
    assert float((gw[77].double().cpu() - e_gw[77]).norm() / e_gw[77].norm()) <= 2.0 ** -8 + 1e-5
    columns = torch.arange(64) != 5
    e_gh = (G[:, keep] @ w[keep].double() + G[:, 77:78] * torch.where(columns, w[77].double(), 0.0))[:, columns]
    assert float((gh.double().cpu()[:, columns] - e_gh).norm() / e_gh.norm()) <= 2.0 ** -7
    assert float(gh[r, 5]) == float("inf")
    # +inf at the target: NaN, as anywhere
    w[77, 5] = float("inf")
    loss, lse = engine.xent_forward(*(x.to(DEV) for x in (h, w, t)))
    assert torch.isnan(loss[r]) and torch.isnan(lse[r])
    assert engine.xent_status() == 0


def test_one_id_alone():
    """A vocabulary of one: the loss is 0 and so are the gradients."""
    from paper_2607_07388_b200 import engine
    h, w = torch.randn((70, 64), device=DEV).bfloat16(), torch.randn((1, 64), device=DEV).bfloat16()
    t = torch.zeros(70, dtype=torch.int32, device=DEV)
    for n in (3, 70):
        loss, lse = engine.xent_forward(h[:n], w, t[:n])
        gh, gw = engine.xent_backward(torch.ones(n, device=DEV), h[:n], w, t[:n], lse)
        z = h[:n].double() @ w[0].double()
        assert not loss.any() and not gh.any() and not gw.any() and float((lse.double() - z).abs().max()) <= 1e-5 * float(z.abs().max())


def sure_rows(seed, n, v, d):
    """Rows whose 1 - p runs from 1e-2 to 1e-6: hidden states along their target's weights, as far as it takes."""
    rng = torch.Generator().manual_seed(seed)
    w = weights(rng, v, d)
    t = torch.randperm(v, generator=rng)[:n].int()
    h = 0.3 * torch.randn((n, d), generator=rng)
    z = h.double() @ w.double().T
    own, along = w[t.long()].double(), w[t.long()].double() @ w.double().T
    want = torch.logspace(-2, -6, n, dtype=torch.float64)
    lo, hi = torch.zeros(n, dtype=torch.float64), torch.full((n,), 20.0, dtype=torch.float64)
    rows = torch.arange(n)
    for _ in range(40):
        k = (lo + hi) / 2
        p = torch.softmax(z + k[:, None] * along, 1)
        p[rows, t.long()] = 0
        more = p.sum(1) > want
        lo, hi = torch.where(more, k, lo), torch.where(more, hi, k)
    h = (h.double() + lo[:, None] * own).bfloat16()
    return h, w, t, torch.rand(n, generator=rng) + 0.5


SURE = [(1, 300, 1024), (40, 2000, 1024), (150, 2000, 1024), (300, 3001, 1024), (40, 2000, 4096), (270, 1200, 4096), (300, 3001, 64)]


@pytest.mark.parametrize("n,v,d", SURE)
def test_loss_of_rows_that_are_sure_of_their_target(n, v, d):
    loss, _ = check_loss(*sure_rows(n + d, n, v, d)[:3])
    assert float(loss.min()) > 0 and (float(loss.min()) < 1e-4 or n == 1)


@pytest.mark.parametrize("n,v,d", SURE)
def test_gradients_of_rows_that_are_sure_of_their_target(n, v, d):
    check(*sure_rows(n + d, n, v, d))


def test_sure_rows_in_several_pieces():
    """4,096 rows x 70,001 ids: the gradient of the logits takes three pieces; the rows' sums run over all of them."""
    from paper_2607_07388_b200 import engine
    h, w, t, g = sure_rows(5, 48, 70_001, 256)
    rng = torch.Generator().manual_seed(6)
    n = 4096
    many_h, many_t, many_g = (0.3 * torch.randn((n, 256), generator=rng)).bfloat16(), torch.full((n,), -1, dtype=torch.int32), torch.ones(n)
    at = torch.randperm(n, generator=rng)[:48].sort().values
    many_h[at], many_t[at], many_g[at] = h, t, g
    hd, wd, td, gd = (x.to(DEV) for x in (many_h, w, many_t, many_g))
    loss, lse = engine.xent_forward(hd, wd, td)
    gh, gw = engine.xent_backward(gd, hd, wd, td, lse)
    e_loss, e_lse, G, e_gh, e_gw = exact(h, w, t, g)
    rel = relative(h, w, e_lse)
    assert bool(((loss.double().cpu()[at] - e_loss).abs() <= e_loss * (rel + 2.0 ** -23)).all())
    # per row, in the 2-norm: G's rounding of the other ids and the result's own, 2^-8 at most each
    for got, want in ((gh.double().cpu()[at], e_gh), (gw.double().cpu()[t.long()], e_gw[t.long()])):
        assert bool(((got - want).norm(dim=1) <= (2.0 ** -7 + 2 * rel) * want.norm(dim=1)).all())


@pytest.mark.parametrize("n,v,d", [(30, 4000, 512), (243, 4000, 512), (600, 4000, 512), (30, 20, 64), (900, 50, 64), (3000, 5000, 128), (70_000, 40, 64)])
def test_one_id_in_half_of_the_rows(n, v, d):
    """A plain mean over unsure rows: G at the target is nearly the same number in every row of an id, and so is its rounding.  Elementwise, within
    half a step of the result and what G's other entries allow."""
    rng = torch.Generator().manual_seed(n + v)
    w = (weights(rng, v, d).float() * 0.01).bfloat16()
    h = torch.randn((n, d), generator=rng).bfloat16()
    t = torch.randint(0, v, (n,), generator=rng).int()
    t[torch.rand(n, generator=rng) < 0.5] = v // 3
    t[:5] = v - 1
    check(h, w, t, torch.full((n,), 1 / n))


def test_identical_rows():
    """The same hidden state and target over and over, as padding that was not masked gives: all errors of one sign."""
    rng = torch.Generator().manual_seed(3)
    w = weights(rng, 700, 256)
    h = torch.randn((1, 256), generator=rng).bfloat16().expand(1500, 256).contiguous()
    check(h, w, torch.full((1500,), 123, dtype=torch.int32), torch.full((1500,), 1 / 1500))


@pytest.mark.parametrize("n", [10, 50, 100, 400])
def test_a_wait_that_runs_out_under_way(n):
    """The MMA issuers give up after their first sum, with copies and MMAs under way, and the other roles find out: NaN in all that has a target, a
    report once, and the next calls as if nothing had been."""
    from paper_2607_07388_b200 import binding as tfe, engine
    rng = torch.Generator().manual_seed(n)
    w, t = weights(rng, 40_000, 1024), torch.randint(-1, 40_000, (n,), generator=rng).int()
    h = torch.randn((n, 1024), generator=rng).bfloat16()
    h, w, t, g = (x.to(DEV) for x in (h, w, t, torch.rand(n, generator=rng) + 0.1))
    loss, lse = engine.xent_forward(h, w, t)
    gh, gw = engine.xent_backward(g, h, w, t, lse)
    assert engine.xent_status() == 0
    tfe.tfe_xent_give_up(2)
    try:
        for _ in range(2):
            bad, bad_lse = engine.xent_forward(h, w, t)
            assert engine.xent_status() != 0 and engine.xent_status() == 0
            bh, bw = engine.xent_backward(g, h, w, t, lse)
            assert engine.xent_status() != 0 and engine.xent_status() == 0
    finally:
        tfe.tfe_xent_give_up(0)
    live = t >= 0
    assert torch.isnan(bad[live]).all() and torch.isnan(bad_lse[live]).all() and not bad[~live].any()
    assert torch.isnan(bh[live]).all() and torch.isnan(bw).all()
    for _ in range(2):
        again = engine.xent_forward(h, w, t)
        grads = engine.xent_backward(g, h, w, t, lse)
        for a, b in zip((*again, *grads), (loss, lse, gh, gw)):
            assert torch.equal(a, b)
    assert engine.xent_status() == 0


@pytest.mark.parametrize("n,v,d", [(4096, 70_001, 64), (20_000, 30_000, 72), (9000, 600, 1032)])
def test_ids_of_a_text(n, v, d):
    """Ids as often as words are, a few in many rows and many in few, over several groups of rows and pieces of the vocabulary, some rows without a
    target and some without a gradient.  The reference runs on the GPU in 64 bits; every target's row of grad_weight by itself, in the 2-norm: its
    own rounding is 2^-8 at most, and what G's other entries are off by, of random signs and 2^-9 in the mean, of their own size.  A row of
    grad_hidden has both roundings, 2^-8 at most each of what is rounded, and of the largest entry where it is one entry."""
    from paper_2607_07388_b200 import engine
    rng = torch.Generator(device=DEV).manual_seed(n)
    w = (torch.randn((v, d), generator=rng, device=DEV) * (2.5 / d ** 0.5)).bfloat16()
    t = (torch.exp(torch.rand(n, generator=rng, device=DEV).double() * math.log(v)) - 1).long().clamp(0, v - 1)
    t = (t * 7919) % v
    h = (torch.randn((n, d), generator=rng, device=DEV) + w[t].float() * torch.rand((n, 1), generator=rng, device=DEV) * 2).bfloat16()
    t = torch.where(torch.rand(n, generator=rng, device=DEV) < 0.1, -1, t).int()
    g = torch.where(torch.rand(n, generator=rng, device=DEV) < 0.1, 0.0, torch.full((n,), 1 / n, device=DEV))
    _, lse = engine.xent_forward(h, w, t)
    gh, gw = engine.xent_backward(g, h, w, t, lse)
    live = ((t >= 0) & (g != 0)).nonzero()[:, 0]
    e_gw = torch.zeros((v, d), dtype=torch.float64, device=DEV)
    size = torch.zeros(v, dtype=torch.float64, device=DEV)       # of a row of grad_weight without the targets' part
    for rows in live.split(1500):
        z, at = h[rows].double() @ w.double().T, t[rows].long()
        k = torch.arange(len(rows), device=DEV)
        p = torch.exp(z - torch.logsumexp(z, 1)[:, None])
        p[k, at] = 0
        size += (p * g[rows].double()[:, None]).square().T @ h[rows].double().square().sum(1)
        p[k, at] = -p.sum(1)
        p *= g[rows].double()[:, None]
        e_gw += p.T @ h[rows].double()
        e_gh = p @ w.double()
        off = (gh[rows].double() - e_gh).norm(dim=1)
        assert bool((off <= 2.0 ** -7 * e_gh.norm(dim=1) + 2.0 ** -8 * p.abs().amax(1)).all()), float((off / e_gh.norm(dim=1)).max())
    ids = t[live].long().unique()
    off = (gw.double() - e_gw)[ids].norm(dim=1)
    assert bool((off <= 2.0 ** -8 * e_gw[ids].norm(dim=1) + 2.0 ** -9 * size[ids].sqrt()).all()), float((off / e_gw[ids].norm(dim=1)).max())
    away = torch.ones(n, dtype=torch.bool, device=DEV)
    away[live] = False
    assert not gh[away].any()
    again = engine.xent_backward(g, h, w, t, lse)
    assert torch.equal(again[0], gh) and torch.equal(again[1], gw) and engine.xent_status() == 0
