"""Distillation of a teacher's top logits, loss and gradient, against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
MASKED = -1e30


def reference(z, ids, t, tau, g=None):
    """(loss, lse, grad) in float64; ids outside [0, V) are no entries, masked logits have probability 0."""
    z, t = z.astype(np.float64), t.astype(np.float64)
    n, v = z.shape
    loss, lse, grad = np.zeros(n), np.full(n, -np.inf), np.zeros((n, v))
    for r in range(n):
        open_ = z[r] > MASKED
        x = np.where(open_, z[r], -np.inf) / tau
        if open_.any():
            lse[r] = x.max() + np.log(np.exp(x - x.max()).sum())
        ok = (ids[r] >= 0) & (ids[r] < v) & (t[r] > -np.inf)
        if not ok.any() or not open_.any():
            continue
        e = t[r][ok] / tau
        q = np.exp(e - e.max())
        q /= q.sum()
        at = ids[r][ok]
        with np.errstate(divide="ignore"):
            loss[r] = tau * tau * sum(qk * (np.log(qk) - x[i] + lse[r]) for qk, i in zip(q, at) if qk > 0)
        if g is not None and g[r] != 0:
            p = np.exp(x - lse[r])
            np.subtract.at(p, at, q)
            grad[r] = g[r] * tau * p
    return loss, lse, grad


def tolerances(z, ids, t, tau, lse, grad, g, kind):
    """How far the results may be off.  A term exp2((z - m) c) carries the rounding of the difference, of c and of the
    product (3 half-steps of an exponent D, weighted by 2^-D: below 3), and ex2's own error of two units in the last
    place; the sum over a row adds a half-step for each addition in a thread's chain, at most V / 32 and a few."""
    v = z.shape[1]
    term = 2.0 ** -22 + 3 * 2.0 ** -24
    tol_lse = term + (v / 32 + 16) * 2.0 ** -24 + np.abs(np.where(np.isfinite(lse), lse, 0)) * 2.0 ** -24
    # the gradient's probability: z c - lse log2(e), each factor rounded, of exponents up to R
    R = max(np.abs(np.where(z > MASKED, z, 0)).max() / tau, np.abs(np.where(np.isfinite(lse), lse, 0)).max())
    rel_p = 2.0 ** -22 + 4 * R * 2.0 ** -24
    p = np.exp(np.where(z > MASKED, z, -np.inf) / tau - np.where(np.isfinite(lse), lse, 0)[:, None])
    q = 2.0 ** -22                                                       # q <= 1, rounded twice
    tol_grad = np.abs(g)[:, None] * tau * (p * rel_p + q) + 2 * HALF_STEP[kind] * np.abs(grad) + 1e-37
    return tol_lse, tol_grad


def make(seed, n, v, k, kind, masked="none", spread=3.0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.standard_normal((n, v)) * spread).astype(np.float32))
    if masked != "none":
        away = torch.from_numpy(rng.random((n, v)) < 0.3)
        z[away] = float("-inf") if masked == "inf" else torch.finfo(TYPES[kind]).min
    z = z.to(TYPES[kind])
    # teacher entries on logits that are not masked, where there are enough
    order = torch.argsort(z.float() + torch.from_numpy(rng.standard_normal((n, v)).astype(np.float32)), dim=1, descending=True)
    ids = order[:, :k].int()
    if ids.shape[1] < k:
        ids = torch.cat([ids, torch.full((n, k - ids.shape[1]), -1, dtype=torch.int32)], 1)
    t = torch.from_numpy((rng.standard_normal((n, k)) * 2).astype(np.float32))
    g = torch.from_numpy(rng.random(n).astype(np.float32) + 0.1)
    return z, ids.contiguous(), t, g


def check(z, ids, t, g, tau, kind, run=None):
    from paper_2607_07388_b200 import engine
    zd, idd, td, gd = (x.to(DEV) for x in (z, ids, t, g))
    loss, lse = engine.distill_forward(zd, idd, td, tau)
    grad = engine.distill_backward(gd, zd, idd, td, lse, tau)
    zn, idn, tn, gn = z.float().numpy(), ids.numpy(), t.numpy(), g.numpy()
    e_loss, e_lse, e_grad = reference(zn, idn, tn, tau, gn)
    tol_lse, tol_grad = tolerances(zn, idn, tn, tau, e_lse, e_grad, gn, kind)
    got_loss, got_lse, got_grad = loss.cpu().numpy(), lse.cpu().numpy(), grad.float().cpu().numpy()
    dead = ~np.isfinite(e_lse)
    assert np.array_equal(got_lse[dead], e_lse[dead])
    assert (np.abs(got_lse[~dead] - e_lse[~dead]) <= tol_lse[~dead]).all()
    far = np.isinf(e_loss)
    assert np.array_equal(got_loss[far], e_loss[far])
    # loss = tau^2 (a sum done in 64 bits + lse)
    off = np.abs(got_loss[~far] - e_loss[~far])
    assert (off <= tau * tau * tol_lse[~far] + 2.0 ** -23 * np.abs(e_loss[~far]) + 1e-30).all()
    assert (np.abs(got_grad - e_grad) <= tol_grad).all(), np.max(np.abs(got_grad - e_grad) / tol_grad)
    return loss, lse, grad


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n,v,k,tau", [(1, 1, 1, 1.0), (3, 2, 1, 2.0), (5, 7, 7, 0.5), (9, 33, 16, 1.0), (17, 2048, 64, 4.0),
                                       (8, 2049, 5, 1.0), (2, 4097, 256, 2.0), (3, 4104, 257, 1.0), (1, 50_001, 1024, 1.0),
                                       (2, 151_936, 64, 1.0), (300, 5003, 3, 2.0), (40, 20_011, 33, 0.7)])
def test_against_formulas(kind, n, v, k, tau):
    check(*make(n + v + k, n, v, k, kind), tau, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("masked", ["inf", "lowest"])
@pytest.mark.parametrize("v", [40, 3001, 70_001])
def test_masked_logits_and_empty_rows(kind, masked, v):
    z, ids, t, g = make(v, 12, v, 8, kind, masked)
    low = float("-inf") if masked == "inf" else torch.finfo(TYPES[kind]).min
    z[0] = low                                      # nothing left to predict
    ids[1] = -1                                     # nothing taught
    ids[2, 1:] = v                                  # one entry, the others outside
    t[3] = float("-inf")                            # entries without weight
    t[4, 2] = float("-inf")
    g[5] = 0.0
    z[6] = low; z[6, v - 1] = 1.0                   # one logit left, at the end
    ids[6] = v - 1
    z[7, int(ids[7, 0])] = low                      # a teacher weight on a masked logit
    ids[8, 1] = ids[8, 0]; ids[8, 5] = ids[8, 0]    # equal ids add up
    ids[9, 0] = -(1 << 31); ids[9, 1] = (1 << 31) - 1
    loss, lse, grad = check(z, ids, t, g, 1.0, kind)
    for r in (0, 1, 3, 5):
        assert not grad[r].any()
    for r in (0, 1, 3):
        assert loss[r] == 0
    assert loss[7] == float("inf") and torch.isfinite(grad[7].float()).all()
    # every entry of row 6 names the only logit left (ln p = 0): what stays is sum q ln q over its entries
    q = torch.softmax(t[6].double(), 0)
    assert abs(float(loss[6]) - float((q * q.log()).sum())) <= 1e-6


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("v,ld,off", [(2001, 2003, 1), (2001, 2048, 3), (40_001, 40_003, 1), (40_000, 40_008, 0), (100, 101, 5)])
def test_strided_rows_and_what_lies_behind_them(kind, v, ld, off):
    """Rows of any alignment; gradient buffers of another alignment; nothing outside the rows is touched."""
    from paper_2607_07388_b200 import engine
    n, k = 6, 9
    z, ids, t, g = make(v + ld, n, v, k, kind)
    store = torch.zeros(n * ld + off, dtype=TYPES[kind], device=DEV)
    zs = torch.as_strided(store, (n, v), (ld, 1), off)
    zs.copy_(z)
    idd, td, gd = ids.to(DEV), t.to(DEV), g.to(DEV)
    plain_loss, plain_lse, plain_grad = check(z, ids, t, g, 1.5, kind)
    loss, lse = engine.distill_forward(zs, idd, td, 1.5)
    _, e_lse, _ = reference(z.float().numpy(), ids.numpy(), t.numpy(), 1.5)
    assert np.abs(lse.cpu().numpy() - e_lse).max() <= 1e-5
    for shift in (off, off + 1):                     # the same alignment as the logits, and another
        behind = torch.full((n * (ld + 1) + off + 1,), 7.0, dtype=TYPES[kind], device=DEV)
        out = torch.as_strided(behind, (n, v), (ld + 1 if shift != off else ld, 1), shift)
        engine.distill_backward(gd, zs, idd, td, plain_lse, 1.5, out=out)
        assert torch.equal(out, plain_grad)
        out.fill_(7.0)
        assert (behind == 7.0).all()
    engine.distill_backward(gd, zs, idd, td, plain_lse, 1.5, out=zs)          # over the logits
    assert torch.equal(zs, plain_grad)
    zs.zero_()
    assert not store.any()


def test_nan_propagates():
    from paper_2607_07388_b200 import engine
    z, ids, t, g = make(1, 4, 9000, 8, "f32")
    z[0, 4000] = float("nan")
    t[1, 3] = float("nan")
    z[2, 17] = float("inf")
    loss, lse = engine.distill_forward(z.to(DEV), ids.to(DEV), t.to(DEV), 1.0)
    assert torch.isnan(lse[0]) and torch.isnan(loss[0]) and torch.isnan(loss[1]) and torch.isnan(loss[2])
    assert torch.isfinite(lse[1]) and torch.isfinite(loss[3])
    grad = engine.distill_backward(g.to(DEV), z.to(DEV), ids.to(DEV), t.to(DEV), lse, 1.0)
    assert torch.isnan(grad[0]).all() and torch.isnan(grad[1][ids[1].long()]).all() and torch.isfinite(grad[3]).all()


@pytest.mark.parametrize("v", [96, 9001])
def test_gradient_against_differences(v):
    """Central differences of the 64-bit loss, and the chain through autograd with a reduction."""
    from paper_2607_07388_b200 import engine
    n, k, tau = 3, 6, 2.0
    z, ids, t, g = make(v, n, v, k, "f32")
    zd = z.to(DEV).requires_grad_()
    (engine.distill_loss(zd, ids.to(DEV), t.to(DEV), tau) * g.to(DEV)).sum().backward()
    got = zd.grad.cpu().numpy()
    rng = np.random.default_rng(5)
    h = 1e-4
    for r in range(n):
        for c in list(rng.integers(0, v, 4)) + [int(ids[r, 0])]:
            zp, zm = z.double().numpy().copy(), z.double().numpy().copy()
            zp[r, c] += h; zm[r, c] -= h
            up, down = (reference(x, ids.numpy(), t.numpy(), tau)[0][r] for x in (zp, zm))
            slope = float(g[r]) * (up - down) / (2 * h)
            assert abs(got[r, c] - slope) <= 1e-6 + 1e-5 * abs(slope), (r, c)


def test_training_step_of_a_projection():
    """W_pref's gradient through the loss: logits = h W^T in fp32, against the formula in 64 bits."""
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(3)
    n, v, d, k = 24, 5001, 64, 16
    h = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(DEV)
    w = torch.from_numpy((rng.standard_normal((v, d)) * 0.2).astype(np.float32)).to(DEV).requires_grad_()
    ids = torch.from_numpy(np.stack([rng.permutation(v)[:k] for _ in range(n)]).astype(np.int32)).to(DEV)
    t = torch.from_numpy(rng.standard_normal((n, k)).astype(np.float32)).to(DEV)
    z = h @ w.T
    engine.distill_loss(z, ids, t, 1.0).mean().backward()
    _, _, dz = reference(z.detach().cpu().numpy(), ids.cpu().numpy(), t.cpu().numpy(), 1.0, np.full(n, 1 / n))
    want = dz.T @ h.double().cpu().numpy()
    got = w.grad.double().cpu().numpy()
    # 24 products of fp32 values of size 1: a few half-steps of the largest term each
    assert np.abs(got - want).max() <= 64 * 2.0 ** -24 * np.abs(dz).max() * float(h.abs().max()) * n


def test_captured_and_replayed_and_other_stream():
    from paper_2607_07388_b200 import engine
    z, ids, t, g = (x.to(DEV) for x in make(8, 5, 30_001, 12, "bf16"))
    loss, lse = engine.distill_forward(z, ids, t, 1.0)
    grad = engine.distill_backward(g, z, ids, t, lse, 1.0)
    zc = torch.zeros_like(z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c_loss, c_lse = engine.distill_forward(zc, ids, t, 1.0)
        c_grad = engine.distill_backward(g, zc, ids, t, c_lse, 1.0)
    for _ in range(2):
        zc.copy_(z)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c_loss, loss) and torch.equal(c_grad, grad)
        zc.zero_()
        graph.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s_loss, s_lse = engine.distill_forward(z, ids, t, 1.0, stream=side)
    s_grad = engine.distill_backward(g, z, ids, t, s_lse, 1.0, stream=side)
    side.synchronize()
    assert torch.equal(s_loss, loss) and torch.equal(s_grad, grad)


def test_rows_beyond_32_bit_offsets():
    """A matrix of more than 2^32 elements: the last row's results are those of the row alone."""
    from paper_2607_07388_b200 import engine
    v, n = 1 << 20, 4100                                                # 4.3e9 bf16 elements
    z = torch.zeros((n, v), dtype=torch.bfloat16, device=DEV)
    zr, idr, tr, gr = make(6, 1, v, 20, "bf16")
    z[-1] = zr[0].to(DEV)
    ids = torch.full((n, 20), -1, dtype=torch.int32, device=DEV)
    ids[-1] = idr[0].to(DEV)
    t = torch.zeros((n, 20), device=DEV)
    t[-1] = tr[0].to(DEV)
    g = torch.ones(n, device=DEV)
    one_loss, one_lse = engine.distill_forward(zr.to(DEV), idr.to(DEV), tr.to(DEV), 1.0)
    loss, lse = engine.distill_forward(z, ids, t, 1.0)
    assert abs(float(loss[-1]) - float(one_loss[0])) <= 1e-5 and abs(float(lse[0]) - np.log(v)) <= 1e-5
    one = engine.distill_backward(g[-1:], zr.to(DEV), idr.to(DEV), tr.to(DEV), one_lse, 1.0)
    lse[-1] = one_lse[0]
    engine.distill_backward(g, z, ids, t, lse, 1.0, out=z)
    assert torch.equal(z[-1], one[0]) and not z[0].any()


def test_empty_batch_and_refusals():
    from paper_2607_07388_b200 import binding as tfe
    from paper_2607_07388_b200 import engine
    z, ids, t, g = (x.to(DEV) for x in make(2, 4, 64, 3, "f32"))
    loss, lse = engine.distill_forward(z[:0], ids[:0], t[:0], 1.0)
    assert loss.shape == (0,) and engine.distill_backward(g[:0], z[:0], ids[:0], t[:0], lse, 1.0).shape == (0, 64)
    for bad in (dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf"))):
        with pytest.raises(tfe.TfeError):
            engine.distill_forward(z, ids, t, **bad)
    for args in ((z.half(), ids, t), (z, ids.long(), t), (z, ids[:3], t), (z, ids, t.bfloat16()), (z.cpu(), ids, t),
                 (z, ids.cpu(), t), (z[0], ids, t), (z.T.contiguous().T, ids, t), (z[:1].expand(4, 64), ids, t)):
        with pytest.raises(ValueError):
            engine.distill_forward(*args, 1.0)
    loss, lse = engine.distill_forward(z, ids, t, 1.0)
    for out in (z.bfloat16(), z[:3], torch.empty((4, 65), device=DEV)):
        with pytest.raises(ValueError):
            engine.distill_backward(g, z, ids, t, lse, 1.0, out=out)
    store = torch.zeros(5 * 64, device=DEV)
    overlap = torch.as_strided(store, (4, 64), (64, 1), 32)
    with pytest.raises(tfe.TfeError):                                   # touches the logits without being them
        engine.distill_backward(g, torch.as_strided(store, (4, 64), (64, 1), 0), ids, t, lse, 1.0, out=overlap)


def test_autograd_sees_what_is_written_over():
    """A tensor that a graph has saved and a call's `out` then overwrites: backward refuses, as after torch's own in-place operations."""
    from paper_2607_07388_b200 import engine
    z, ids, t, g = (x.to(DEV) for x in make(3, 4, 200, 3, "f32"))
    zr = z.clone().requires_grad_()
    loss = engine.distill_loss(zr, ids, t, 1.0)
    _, lse = engine.distill_forward(zr.detach(), ids, t, 1.0)
    engine.distill_backward(g, zr.detach(), ids, t, lse, 1.0, out=zr.detach())
    with pytest.raises(RuntimeError):
        loss.sum().backward()
    zr = z.clone().requires_grad_()
    loss = engine.distill_loss(zr, ids, t, 1.0)
    a, s = engine.quantize_fp8(torch.ones((4, 64), device=DEV))
    w, ws = engine.quantize_fp8(torch.ones((200, 64), device=DEV), 128)
    engine.matmul_fp8(a, s, w, ws, out=zr.detach())
    with pytest.raises(RuntimeError):
        loss.sum().backward()
    with torch.inference_mode():
        z2 = z.clone()
        _, lse = engine.distill_forward(z2, ids, t, 1.0)
        want = engine.distill_backward(g, z2, ids, t, lse, 1.0)
        assert torch.equal(engine.distill_backward(g, z2, ids, t, lse, 1.0, out=z2), want)
    engine.distill_backward(g, z, ids, t, lse.clone(), 1.0, out=z)          # outside, of an ordinary tensor
    assert torch.equal(z, want)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n,v", [(9, 300), (4, 20_000), (400, 20_001), (4, 150_000)])
def test_logits_far_from_zero(kind, n, v):
    """Rows whose logits are so large against tau that fp32 holds z / tau to whole units only, or not at all: the loss is a
    difference and keeps its precision.  Among them rows that a mask of -1e10 has left nothing of."""
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(n + v)
    k = 6
    for size, tau in ((1e6, 1.0), (3e7, 1.0), (1e10, 0.5), (1e10, 1000.0), (3e4, 1e-6), (1e20, 3.0), (2e38, 1.0), (3e38, 1e-6), (3e38, 0.7)):
        t = torch.tensor(size, dtype=torch.float32).to(TYPES[kind])
        steps = [t]                                     # the largest logits: a few steps of the type apart
        for _ in range(4):
            steps.append(torch.nextafter(steps[-1], torch.tensor(0.0, dtype=TYPES[kind])))
        steps = torch.stack(steps)
        z = steps[torch.from_numpy(rng.integers(0, 5, (n, v)))]
        if size < 1e30:                                 # (below -1e30 they would be masked ones)
            z[1::2] = -z[1::2]
        z[0], z[1] = z[0, 0].clone(), z[1, 0].clone()   # equal logits
        z[2, : v // 2] = torch.finfo(TYPES[kind]).min
        z[3, v // 3:] = float("-inf")
        ids = torch.from_numpy(rng.integers(0, v // 3, (n, k)).astype(np.int32)) + v // 2 * (torch.arange(n) == 2)[:, None].int()
        te = torch.from_numpy(rng.standard_normal((n, k)).astype(np.float32))
        loss, lse = engine.distill_forward(z.to(DEV), ids.to(DEV), te.to(DEV), tau)
        # the definition, relative to the largest logit: differences of logits are exact in 64 bits
        zd = z.to(DEV).double()
        d = torch.where(zd > MASKED, zd, float("-inf"))
        top = d.amax(1, keepdim=True)
        d = (d - top) / tau
        norm = torch.log(torch.exp(d).sum(1))
        q = torch.softmax(te.to(DEV).double() / tau, 1)
        terms = torch.where(q > 0, q * (torch.log(q) - d.gather(1, ids.to(DEV).long()) + norm[:, None]), 0.0)
        want = tau * tau * terms.sum(1)
        # the sum: as in `tolerances`; the terms are 64-bit numbers of the size of z / tau, where q-weighted ones cancel
        far = float(top.abs().max()) / tau
        tol = tau * tau * (2.0 ** -22 + 3 * 2.0 ** -24 + (v / 32 + 16) * 2.0 ** -24 + (k + 8) * 2.0 ** -52 * far) + 2.0 ** -23 * want.abs()
        got = loss.double()
        assert not torch.isnan(got).any() and ((got - want).abs() <= tol).all(), (size, tau, float(((got - want).abs() / tol).max()))
        e_lse = top[:, 0] / tau + norm
        assert ((lse.double() - e_lse).abs() <= 2.0 ** -24 * e_lse.abs() + tol / tau ** 2)[e_lse.abs() < 3.4e38].all()
    z[0, 7] = float("inf")
    loss, lse = engine.distill_forward(z.to(DEV), ids.to(DEV), te.to(DEV), tau)
    assert torch.isnan(loss[0]) and torch.isnan(lse[0]) and not torch.isnan(loss[1:]).any()
