"""A training step of the memory path as a program makes it: memory rows looked up by token ids, injected between two norms with a learned
gate, cross entropy of the next token against the projection, the gradients of all that is trained, clipped together."""
import numpy as np
import pytest
import torch

from paper_2607_07388_b200 import synth

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def make_step():
    from paper_2607_07388_b200.engine import Engram, bf16_tensor_from_bits
    w = synth.config(1, residency="hot_host_ssd", gpu_slots=16_000)
    tb = synth.make_table(w)
    eng = Engram(tb.phrase_tokens, tb.phrase_len, tb.init_slot, bf16_tensor_from_bits(synth.make_rows_np(w, tb), DEV), vocab=w.vocab, orders=w.orders,
                 load_factor=w.load_factor)
    tokens = torch.from_numpy(synth.make_queries(w, tb)).to(DEV)
    rng = torch.Generator(device=DEV).manual_seed(3)
    d, vocab = w.d, 5003
    target = (tokens.flatten().long() * 7 % vocab).int()
    target[::9] = -1                                # padding
    leaves = dict(h=torch.randn((w.Q, d), generator=rng, device=DEV).bfloat16(), gate=torch.randn((w.Q, d), generator=rng, device=DEV).bfloat16(),
                  post=1 + 0.1 * torch.randn(d, generator=rng, device=DEV), next=1 + 0.1 * torch.randn(d, generator=rng, device=DEV),
                  proj=(torch.randn((vocab, d), generator=rng, device=DEV) * 2 / d ** 0.5).bfloat16())
    return eng, tokens, target, leaves


def memory(eng, tokens, like):
    """m itself: the lookup's rows injected into zeros."""
    got = eng.lookup_inject(tokens, torch.zeros_like(like), lam=1.0)
    return got.out, got.flags


def test_training_step():
    from paper_2607_07388_b200 import engine
    eng, tokens, target, leaves = make_step()
    m, flags = memory(eng, tokens, leaves["h"])
    assert int((flags == 1).sum()) > 0 and bool((m[flags.flatten() != 1] == 0).all())
    x = {k: v.clone().requires_grad_() for k, v in leaves.items()}
    out, normed = engine.normed_inject(x["h"], m, x["post"], x["next"], x["gate"], sigmoid=True, lam=0.5)
    loss = engine.linear_cross_entropy(normed, x["proj"], target)
    (loss.sum() / (target >= 0).sum()).backward()
    # the same in torch's own operations, rounded at the same places
    y = {k: v.clone().float().requires_grad_() for k, v in leaves.items()}
    mf = m.float()
    u = y["h"] + 0.5 * torch.sigmoid(y["gate"]) * (y["post"] * mf * torch.rsqrt((mf * mf).mean(1, keepdim=True) + 1e-6))
    n = (y["next"] * u * torch.rsqrt((u * u).mean(1, keepdim=True) + 1e-6)).bfloat16().float()
    live = target >= 0
    z = (n.double() @ y["proj"].double().T)[live]
    e_loss = torch.logsumexp(z, 1) - z.gather(1, target[live].long()[:, None])[:, 0]
    (e_loss.sum() / live.sum()).backward()
    # normed may round to the other of two bf16 numbers here and there: 2^-8 of an element, in few of d
    assert float((loss.detach()[live].double() - e_loss.detach()).abs().max()) <= 2.0 ** -7 and not loss[~live].any()
    grads = {k: v.grad for k, v in x.items()}
    for k, v in grads.items():
        want = y[k].grad.double()
        # roundings of G, of the gradient that arrives at normed, and of the result, each 2^-8 at most
        assert float((v.double() - want).norm() / want.norm()) <= 3 * 2.0 ** -8, k
    total = float(sum((v.double() ** 2).sum() for v in grads.values()) ** 0.5)
    before = {k: v.clone() for k, v in grads.items()}
    norm = engine.clip_grad_norm(list(grads.values()), 0.5 * total)
    assert abs(float(norm) - total) <= 1e-6 * total
    for k, v in grads.items():
        assert float((v.double() - 0.5 * before[k].double()).norm() / before[k].double().norm()) <= 2.0 ** -8
    assert engine.xent_status() == 0
    eng.close()


def test_training_step_captured():
    """Lookup, both passes and clipping in one CUDA graph, replayed on other contents: to the bit what the calls give by themselves."""
    from paper_2607_07388_b200 import binding as tfe, engine
    eng, tokens, target, leaves = make_step()
    zeros = torch.zeros_like(leaves["h"])

    def step(tok, tgt, x):
        m = torch.empty_like(zeros)
        tfe.tfe_lookup_inject(eng.ctx, tok, tok.shape[0], tok.shape[1], 0, zeros, m)
        out, normed = engine.normed_inject_forward(x["h"], m, x["post"], x["next"], x["gate"], sigmoid=True, lam=0.5)
        loss, lse = engine.xent_forward(normed, x["proj"], tgt)
        gn, gproj = engine.xent_backward(torch.full_like(loss, 1 / 64), normed, x["proj"], tgt, lse)
        grads = [*engine.normed_inject_backward(None, gn, x["h"], m, x["post"], x["next"], x["gate"], sigmoid=True, lam=0.5), gproj]
        norm = engine.clip_grad_norm(grads, 1e-3)
        return [loss, norm, *grads]

    others = {k: v.flip(0).contiguous() for k, v in leaves.items()}
    inputs = [(tokens, target, leaves), (tokens.flip(0).contiguous(), target.flip(0).contiguous(), others)]
    want = [[t.clone() for t in step(*i)] for i in inputs]
    assert float(want[0][1]) > 1e-3
    held = (tokens.clone(), target.clone(), {k: v.clone() for k, v in leaves.items()})
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = step(*held)
    for k in (1, 0, 1):
        held[0].copy_(inputs[k][0]); held[1].copy_(inputs[k][1])
        for name, v in held[2].items():
            v.copy_(inputs[k][2][name])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(made, want[k]):
            assert torch.equal(a, b)
    del graph
    eng.close()


def test_example_runs():
    """An example as in the documentation: it runs, and every trained tensor gets a gradient that is finite and not zero."""
    from paper_2607_07388_b200 import engine
    eng, tokens, target, leaves = make_step()
    m, _ = memory(eng, tokens, leaves["h"])
    x = {k: v.clone().requires_grad_() for k, v in leaves.items() if k != "h"}
    for _ in range(2):
        _, normed = engine.normed_inject(leaves["h"], m, x["post"], x["next"], x["gate"], sigmoid=True, lam=0.5)
        loss = engine.linear_cross_entropy(normed, x["proj"], target)
        grads = torch.autograd.grad(loss.sum() / (target >= 0).sum(), list(x.values()))
        assert all(bool(torch.isfinite(g).all()) and bool(g.any()) for g in grads)
        engine.clip_grad_norm(grads, 1.0)
        with torch.no_grad():
            for p, g in zip(x.values(), grads):
                p -= 0.1 * g
    eng.close()
