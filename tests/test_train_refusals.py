"""Refusals of the calls that train the memory path: found on the host, before any device call (nothing here needs a GPU)."""
import ctypes as C
from array import array

import pytest

P = 1 << 20                                 # an address that is never touched


@pytest.fixture(scope="module")
def tfe():
    from paper_2607_07388_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def test_cross_entropy(tfe):
    L = tfe.lib()
    far = 1 << 30

    def forward(h=P, ld_h=64, N=4, w=2 * P, ld_w=64, V=100, d=64, t=3 * P, loss=4 * P, lse=5 * P, ws=far, size=1 << 40):
        return L.tfe_xent_forward(h, ld_h, N, w, ld_w, V, d, t, loss, lse, ws, size, None)

    def backward(h=P, ld_h=64, N=4, w=2 * P, ld_w=64, V=100, d=64, t=3 * P, lse=5 * P, g=6 * P, gh=7 * P, ld_gh=64, gw=8 * P, ld_gw=64, ws=far, size=1 << 40):
        return L.tfe_xent_backward(h, ld_h, N, w, ld_w, V, d, t, lse, g, gh, ld_gh, gw, ld_gw, ws, size, None)

    both = [dict(N=-1), dict(N=tfe.XENT_MAX_ROWS + 1), dict(V=0), dict(V=tfe.XENT_MAX_ROWS + 1), dict(d=0), dict(d=60), dict(d=7), dict(d=tfe.XENT_MAX_COLS + 8, ld_h=1 << 20, ld_w=1 << 20),
            dict(ld_h=56), dict(ld_h=68), dict(ld_h=1 << 40), dict(ld_w=56), dict(ld_w=66), dict(h=None), dict(h=P + 8), dict(w=None), dict(w=2 * P + 2), dict(t=None), dict(t=3 * P + 2),
            dict(lse=None), dict(lse=5 * P + 1), dict(ws=None), dict(ws=far + 16)]
    for kw in both + [dict(loss=None), dict(loss=4 * P + 2), dict(loss=P), dict(lse=2 * P + 64), dict(loss=3 * P), dict(loss=5 * P), dict(lse=far + 512), dict(h=far + 64), dict(t=far)]:
        assert forward(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    for kw in both + [dict(g=None), dict(g=6 * P + 2), dict(gh=None, gw=None), dict(gh=7 * P + 8), dict(gw=8 * P + 4), dict(ld_gh=56), dict(ld_gw=60), dict(gh=P), dict(gw=2 * P),
                      dict(gh=2 * P + 128), dict(gw=P + 16), dict(gh=8 * P + 16), dict(gw=3 * P), dict(gh=far + 1024), dict(gw=far), dict(gh=5 * P), dict(gw=6 * P), dict(w=far + 128), dict(g=far)]:
        assert backward(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    need = tfe.tfe_xent_forward_workspace_bytes(4, 100, 64), tfe.tfe_xent_backward_workspace_bytes(4, 100, 64)
    assert min(need) > 0
    assert forward(size=need[0] - 1) == tfe.TFE_ERR_CAPACITY and backward(size=need[1] - 1) == tfe.TFE_ERR_CAPACITY
    assert forward(N=0, h=None, t=None, loss=None, lse=None, ws=None, size=0) == tfe.TFE_OK
    assert backward(N=0, h=None, t=None, lse=None, g=None, gh=7 * P, gw=None, ws=None, size=0) == tfe.TFE_OK
    for bad in ((-1, 100, 64), (4, 0, 64), (4, 100, 12)):
        assert tfe.tfe_xent_forward_workspace_bytes(*bad) == -1 and tfe.tfe_xent_backward_workspace_bytes(*bad) == -1
    # the workspace holds a piece of the logits' gradient and no more: far less than the logits of a training batch
    assert tfe.tfe_xent_backward_workspace_bytes(8192, 151_936, 1024) < 8192 * 151_936 * 2 / 3
    assert tfe.tfe_xent_forward_workspace_bytes(32_768, 151_936, 1024) < 32_768 * 151_936 * 2 / 40
    assert L.tfe_xent_status(None, None) == tfe.TFE_ERR_INVALID_ARG


def test_injection_between_norms(tfe):
    L = tfe.lib()
    ok = dict(dtype=1, Q=4, d=32, gate_kind=2, sigmoid=0, weight_dtype=1, h=P, m=2 * P, gate=3 * P, ld_h=32, ld_m=32, ld_gate=32, post_weight=4 * P, next_weight=5 * P, lam=1.0, eps=1e-6)

    def params(**kw):
        return C.byref(tfe.TfeInjectNormParams(**(ok | kw)))

    def forward(out=6 * P, ld_out=32, normed=7 * P, ld_normed=32, **kw):
        return L.tfe_inject_norm_forward(params(**kw), out, ld_out, normed, ld_normed, None)

    made = dict(grad_out=8 * P, grad_normed=9 * P, ld_grad_out=32, ld_grad_normed=32, grad_h=10 * P, grad_m=11 * P, grad_gate=12 * P, ld_grad_h=32, ld_grad_m=32, ld_grad_gate=32,
                grad_post=13 * P, grad_next=14 * P)

    def backward(grads=None, ws=15 * P, size=1 << 30, **kw):
        return L.tfe_inject_norm_backward(params(**kw), C.byref(tfe.TfeInjectNormGrads(**(made | (grads or {})))), ws, size, None)

    both = [dict(dtype=2), dict(weight_dtype=-1), dict(Q=-1), dict(Q=tfe.ROWS_MAX + 1), dict(d=0), dict(d=tfe.INJECT_NORM_MAX_COLS + 1, ld_h=1 << 20, ld_m=1 << 20, ld_gate=1 << 20),
            dict(gate_kind=3), dict(gate_kind=-1), dict(eps=-1e-6), dict(eps=2.0), dict(eps=float("nan")), dict(lam=float("inf")), dict(lam=float("nan")), dict(h=None), dict(h=P + 2),
            dict(m=None), dict(gate=None), dict(gate=3 * P + 1), dict(gate_kind=1, gate=3 * P + 2), dict(ld_h=31), dict(ld_m=8), dict(ld_gate=31), dict(ld_h=1 << 40), dict(post_weight=None),
            dict(next_weight=5 * P + 2)]
    for kw in both + [dict(out=None), dict(normed=None), dict(out=6 * P + 2), dict(ld_out=31), dict(ld_normed=1), dict(out=2 * P), dict(out=P, ld_out=40), dict(out=P + 4), dict(normed=P),
                      dict(normed=6 * P), dict(normed=3 * P), dict(out=4 * P), dict(normed=5 * P)]:
        assert forward(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    for kw in both:
        assert backward(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    for g in (dict(grad_out=None, grad_normed=None), dict(grad_out=8 * P + 1), dict(ld_grad_normed=31), dict(grad_h=10 * P + 2), dict(ld_grad_m=31), dict(grad_gate=12 * P + 3), dict(ld_grad_gate=4),
              dict(grad_post=13 * P + 2), dict(grad_next=14 * P + 1), dict(grad_h=P), dict(grad_m=8 * P), dict(grad_h=11 * P), dict(grad_post=14 * P), dict(grad_gate=3 * P), dict(grad_next=15 * P)):
        assert backward(g) == tfe.TFE_ERR_INVALID_ARG, g
    assert backward(gate_kind=0) == tfe.TFE_ERR_INVALID_ARG         # a gradient for a gate that is not there
    assert backward(ws=None) == tfe.TFE_ERR_INVALID_ARG
    assert backward(size=tfe.tfe_inject_norm_workspace_bytes(4, 32) - 1) == tfe.TFE_ERR_CAPACITY
    assert forward(Q=0, h=None, m=None, gate=None, out=None, normed=None) == tfe.TFE_OK
    assert L.tfe_inject_norm_forward(None, P, 32, P, 32, None) == L.tfe_inject_norm_backward(None, None, P, 0, None) == tfe.TFE_ERR_INVALID_ARG
    assert backward(dict(grad_post=None, grad_next=None), Q=0) == tfe.TFE_OK
    assert tfe.tfe_inject_norm_workspace_bytes(-1, 32) == tfe.tfe_inject_norm_workspace_bytes(4, 0) == -1


def test_clipping(tfe):
    L = tfe.lib()

    def clip(at=(P, 2 * P), out=None, n=(100, 50), kind=(1, 0), count=2, max_norm=1.0, norm=3 * P, ws=4 * P, size=1 << 30):
        lists = [None if x is None else array(c, x) for x, c in ((at, "Q"), (out, "Q"), (n, "q"), (kind, "i"))]
        return L.tfe_clip_grad_norm(*(None if x is None else x.buffer_info()[0] for x in lists), count, max_norm, norm, ws, size, None)

    for kw in (dict(count=-1), dict(count=tfe.CLIP_MAX_TENSORS + 1), dict(at=None), dict(n=None), dict(kind=None), dict(norm=None), dict(norm=3 * P + 2), dict(max_norm=-1.0), dict(max_norm=float("nan")),
               dict(n=(-1, 5)), dict(n=(1 << 41, 5)), dict(kind=(2, 0)), dict(at=(P + 2, 2 * P)), dict(at=(0, 2 * P)), dict(at=(P, 2 * P + 1)), dict(out=(5 * P, 0)), dict(out=(5 * P + 1, 6 * P)),
               dict(ws=None), dict(ws=4 * P + 4), dict(at=(P, P)), dict(at=(P, P + 396)), dict(at=(P, 3 * P)), dict(norm=P + 40), dict(at=(P, 4 * P)), dict(out=(5 * P, 5 * P + 396)),
               dict(out=(5 * P, P)), dict(out=(P + 4, 6 * P)), dict(out=(2 * P, 6 * P))):
        assert clip(**kw) == tfe.TFE_ERR_INVALID_ARG, kw
    assert clip(size=tfe.tfe_clip_workspace_bytes(2) - 1) == tfe.TFE_ERR_CAPACITY
    assert tfe.tfe_clip_workspace_bytes(-1) == -1 and tfe.tfe_clip_workspace_bytes(2000) > tfe.tfe_clip_workspace_bytes(2) > 0


def test_describing_tensors(tfe):
    """On the CPU every tensor is refused for where it is; what describes it runs all the same."""
    import torch
    for t in (torch.ones(3), torch.nn.Parameter(torch.ones(2, 2)), torch.ones(4, dtype=torch.float64), torch.ones(4, 4).t()):
        at, numel, kinds, device, reason = tfe.tfe_describe_tensors([t])
        assert reason == 1 and len(at) == len(numel) == len(kinds) == 1
    with pytest.raises(RuntimeError):
        tfe.tfe_describe_tensors([torch.ones(3).to_sparse()])
    from paper_2607_07388_b200 import engine
    for bad in ([], [None], [torch.ones(3), 1.0], [torch.ones(3)], [torch.ones(3).to_sparse()], [torch.ones(3, device="meta")], torch.ones(3)):
        with pytest.raises(ValueError):
            engine.grad_norm(bad)
        with pytest.raises(ValueError):
            engine.clip_grad_norm(bad, 1.0)
    L = tfe.lib()
    assert L.tfe_describe_tensors(None, None, None, 1, None, None, None, None, None) == tfe.TFE_ERR_INVALID_ARG
