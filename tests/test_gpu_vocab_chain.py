"""The calls at the vocabulary axis in the order a program makes them: hidden states to logits in 8 bits, a draw, and the lookup
of what was drawn; a teacher's top tokens to the loss and gradient of a predictor."""
import numpy as np
import pytest
import torch

from paper_2607_07388_b200 import synth

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def test_decode_step_from_hidden_states_to_injection():
    """Every step: logits (8-bit head), one draw per sequence, the drawn token behind the prefix, lookup and injection against
    the oracle; the draw against the definition on the same logits.  A finished sequence's row is masked: it draws -1, which the
    lookup takes as padding.  The whole step replayed from a CUDA graph gives the same."""
    import parity_harness as H
    from paper_2607_07388_b200.engine import QuantizedHead, sample_tokens
    from test_gpu_sample import draw64
    w = synth.config(2, n_phrases=60_000, gpu_slots=30_000, B=24)
    tb, pr = H.pair_from_workload(w)
    B, V, dh = w.B, w.vocab, 64
    rng = np.random.default_rng(21)
    Wf = (rng.standard_normal((V, dh)) * 0.3).astype(np.float32)
    head = QuantizedHead(torch.from_numpy(Wf).to(torch.bfloat16).to(DEV))
    pos = tb.safe_len // 2 + 7 * np.arange(B)
    tokens = torch.from_numpy(np.stack([tb.stream[p - 2:p + 1] for p in pos]).astype(np.int32)).to(DEV)
    h_main = synth.make_hidden_np(w, Q=B)
    hits = 0
    for step in range(3):
        nxt = tb.stream[pos + 1 + step]
        hidden = torch.from_numpy(4 * np.sign(Wf[nxt]) + rng.standard_normal((B, dh)).astype(np.float32)).to(torch.bfloat16).to(DEV)
        u = torch.from_numpy(rng.random(B).astype(np.float32)).to(DEV)
        T = torch.full((B,), 0.7, device=DEV)
        k = torch.full((B,), 40, dtype=torch.int32, device=DEV)
        p = torch.full((B,), 0.9, device=DEV)
        z = head.logits(hidden)
        z[B - 1] = float("-inf")
        token, prob = sample_tokens(z, u, temperature=T, top_k=k, top_p=p)
        zn, un = z.double().cpu().numpy(), u.double().cpu().numpy()
        for r in range(B):
            e_token, e_prob = draw64(zn[r], un[r], float(np.float32(0.7)), 40, float(np.float32(0.9)))
            assert int(token[r]) == e_token and abs(float(prob[r]) - e_prob) <= 2.0 ** -23 * e_prob + 1e-10
        assert int(token[B - 1]) == -1
        tokens = torch.cat([tokens[:, 1:], token[:, None]], 1).contiguous()
        _, ref, _ = pr.run_and_compare(tokens.cpu().numpy(), h_main, q_start=2)
        hits += int((ref.flags == 1).sum())
        assert ref.flags[B - 1] == 0
    assert hits > 0
    # the last step once more, captured
    from paper_2607_07388_b200 import binding as tfe
    h_gpu = pr.hidden_to_gpu(h_main)
    before = tokens.clone()
    want = pr.eng.lookup_inject(before, h_gpu, q_start=2).out.clone()
    hid_c, u_c, tok_c, out_c = torch.zeros_like(hidden), torch.zeros_like(u), before.clone(), torch.empty_like(h_gpu)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zc = head.logits(hid_c)
        zc[B - 1].fill_(float("-inf"))
        drawn, _ = sample_tokens(zc, u_c, temperature=T, top_k=k, top_p=p)
        tok_c[:, 2] = drawn
        tfe.tfe_lookup_inject(pr.eng.ctx, tok_c, B, 3, 2, h_gpu, out_c)
    for _ in range(2):
        hid_c.copy_(hidden); u_c.copy_(u); tok_c.zero_(); tok_c[:, :2] = before[:, :2]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok_c, before) and torch.equal(out_c, want)
        hid_c.zero_()
        graph.replay()
    pr.close()


def test_teacher_top_tokens_to_gradient():
    """The teacher's head gives its top tokens and probabilities, their logarithms are the teacher logits; the predictor's gradient
    reaches its projection.  Against the formula in 64 bits."""
    from paper_2607_07388_b200.engine import EarlyExitHead, bf16_tensor_from_bits, distill_loss
    from test_gpu_distill import reference
    rng = np.random.default_rng(5)
    V, d, B, K = 5003, 128, 24, 32
    teacher = EarlyExitHead(bf16_tensor_from_bits(synth.f32_to_bf16_bits((rng.standard_normal((V, d)) * 0.2).astype(np.float32)), DEV), max_batch=B)
    h = torch.from_numpy(rng.standard_normal((B, d)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    ids, prob = teacher.topk(h, K)
    assert teacher.status() == 0
    t = prob.log()
    w = torch.from_numpy((rng.standard_normal((V, d)) * 0.1).astype(np.float32)).to(DEV).requires_grad_()
    z = h.float() @ w.T
    weight = torch.from_numpy(rng.random(B).astype(np.float32)).to(DEV)
    weight[3] = 0.0
    loss = distill_loss(z, ids, t, 1.5)
    (loss * weight).sum().backward()
    e_loss, _, dz = reference(z.detach().cpu().numpy(), ids.cpu().numpy(), t.cpu().numpy(), 1.5, weight.cpu().numpy())
    # logits of size 5 and sums of 5,003 terms: a few units of 2^-24 of lse = 9, times tau^2
    assert np.abs(loss.detach().cpu().numpy() - e_loss).max() <= 2e-5
    want = dz.T @ h.double().cpu().numpy()
    got = w.grad.double().cpu().numpy()
    assert np.abs(got - want).max() <= 64 * 2.0 ** -24 * np.abs(dz).max() * float(h.abs().max()) * B
    teacher.close()


def test_training_step_captured():
    """Forward and gradient in one CUDA graph, replayed with other contents."""
    from paper_2607_07388_b200.engine import distill_loss
    rng = np.random.default_rng(6)
    n, v, k = 6, 3001, 5
    z = torch.from_numpy(rng.standard_normal((n, v)).astype(np.float32)).to(DEV)
    ids = torch.from_numpy(rng.integers(0, v, (n, k)).astype(np.int32)).to(DEV)
    t = torch.from_numpy(rng.standard_normal((n, k)).astype(np.float32)).to(DEV)
    zr = z.clone().requires_grad_()
    want, = torch.autograd.grad(distill_loss(zr, ids, t, 1.0).sum(), zr)
    zc = torch.zeros_like(z).requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(distill_loss(zc, ids, t, 1.0).sum(), zc)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grad, = torch.autograd.grad(distill_loss(zc, ids, t, 1.0).sum(), zc)
    for _ in range(2):
        with torch.no_grad():
            zc.copy_(z)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, want)
        with torch.no_grad():
            zc.zero_()
        graph.replay()
