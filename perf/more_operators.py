"""Cases of the operators that train the memory path, with their plain forms.

Three families: softmax cross entropy of hidden states against a vocabulary projection, without the logits
(``xent_loss``, and ``xent_step`` with the gradients of both), an injection with a norm before and after its gate
(``inject`` and ``inject_grad``), and the norm of many gradients with clipping (``clip``).  ``own`` selects who
computes: False, elementary torch operations; True, the package.
"""
import math

import torch

own = False

VOCAB, WIDTH = 151_936, 1024       # the vocabulary and row width of the benchmark's tables
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6


def listed():
    return [
        # one position scored against the whole vocabulary: reads every weight for one row
        dict(name="xent_loss_1", op="xent_loss", rows=1, vocab=VOCAB, d=WIDTH, ignored=0.0),
        # an evaluation batch: bound by the arithmetic
        dict(name="xent_loss_2048", op="xent_loss", rows=2048, vocab=VOCAB, d=WIDTH, ignored=0.05),
        # odd sizes everywhere, a small vocabulary: the end of a training batch
        dict(name="xent_step_33", op="xent_step", rows=33, vocab=32_003, d=1000, ignored=0.1),
        # a fine-tuning step on few sequences: the projection and its gradient pass through memory
        dict(name="xent_step_256", op="xent_step", rows=256, vocab=VOCAB, d=WIDTH, ignored=0.0),
        # a training step whose prompts teach nothing
        dict(name="xent_step_4096", op="xent_step", rows=4096, vocab=VOCAB, d=WIDTH, ignored=0.3),
        # one decoded token, a learned scalar gate: nothing but latency
        dict(name="inject_1", op="inject", rows=1, d=WIDTH, dtype="bf16", gate="scalar", sigmoid=True, weights="f32"),
        # the benchmark's prefill, 8 x 4,096 positions, a gate for every channel
        dict(name="inject_32768", op="inject", rows=32_768, d=WIDTH, dtype="bf16", gate="vector", sigmoid=True, weights="bf16"),
        dict(name="inject_grad_7", op="inject_grad", rows=7, d=1001, dtype="f32", gate="scalar", sigmoid=False, weights="f32"),
        dict(name="inject_grad_32768", op="inject_grad", rows=32_768, d=WIDTH, dtype="bf16", gate="vector", sigmoid=True, weights="bf16"),
        # the gradients of the norms and the gate's projection of one layer
        dict(name="clip_4", op="clip", kind="layer", tensors=4, total=1 << 17, dtype="f32"),
        # a model's many tensors, small and large, of both types
        dict(name="clip_400", op="clip", kind="model", tensors=400, total=1 << 27, dtype="bf16"),
        # the projection's gradient: one tensor of 311 MB
        dict(name="clip_projection", op="clip", kind="one", tensors=1, total=VOCAB * WIDTH, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["xent_loss", "xent_step", "inject", "inject_grad", "clip"])
    dtype = rng.choice(["bf16", "f32"])
    if op in ("xent_loss", "xent_step"):
        vocab = _log(rng, 100, 262_144)
        d = 8 * _log(rng, 8, 512)
        rows = _log(rng, 1, max(1, min(16_384, 4096 * VOCAB // vocab, 2048 * VOCAB * WIDTH // (vocab * d))))
        return dict(op=op, rows=rows, vocab=vocab, d=d, ignored=rng.choice([0.0, 0.05, 0.5]))
    if op in ("inject", "inject_grad"):
        d = _log(rng, 16, 8192)
        return dict(op=op, rows=_log(rng, 1, min(65_536, 16_384 * WIDTH // d)), d=d, dtype=dtype, gate=rng.choice(["none", "scalar", "vector"]),
                    sigmoid=rng.choice([True, False]), weights=rng.choice(["bf16", "f32"]))
    kind = rng.choice(["layer", "model", "one"])
    tensors = 1 if kind == "one" else _log(rng, 2, 1000)
    return dict(op=op, kind=kind, tensors=tensors, total=_log(rng, 1000 * tensors, VOCAB * WIDTH // 2), dtype=dtype)


# ---- inputs ---------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, s = case["op"], dict(op=case["op"])

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if op in ("xent_loss", "xent_step"):
        n, v, d = case["rows"], case["vocab"], case["d"]
        s["weight"] = torch.empty((v, d), dtype=torch.bfloat16, device="cuda")
        for at in range(0, v, 32_768):
            s["weight"][at:at + 32_768] = randn(min(32_768, v - at), d) * (2.5 / math.sqrt(d))       # logits spread over 2.5
        target = torch.randint(0, v, (n,), generator=g, device="cuda")
        # hidden states that know their target more or less
        s["hidden"] = (randn(n, d) + s["weight"][target].float() * (rand(n, 1) * 2.5)).to(torch.bfloat16)
        away = rand(n) < case["ignored"]
        away[0] = False
        s["target"] = target.masked_fill(away, -1).int()
        if op == "xent_step":
            s["grad_loss"] = torch.where(away, 0.0, 1.0 / (~away).sum()) * (0.5 + rand(n))              # a weighted mean
    elif op in ("inject", "inject_grad"):
        n, d, dt = case["rows"], case["d"], DTYPES[case["dtype"]]
        s["h"] = (randn(n, d) * torch.exp(0.5 * randn(n, 1))).to(dt)
        s["m"] = (randn(n, d) * (0.05 * torch.exp(randn(n, 1)))).to(dt)                                   # memory rows
        if n > 2:
            s["m"][n // 2] = 0                                                                             # a position without a phrase
        s["gate"] = {"none": None, "scalar": randn(n), "vector": randn(n, d).to(dt)}[case["gate"]]
        s["post_weight"] = (1 + 0.2 * randn(d)).to(DTYPES[case["weights"]])
        s["next_weight"] = (1 + 0.2 * randn(d)).to(DTYPES[case["weights"]])
        s["sigmoid"], s["lam"] = case["sigmoid"], 0.75
        if op == "inject_grad":
            s["grad_out"], s["grad_normed"] = (randn(n, d) / n).to(dt), (randn(n, d) / n).to(dt)
    else:
        k, total = case["tensors"], case["total"]
        if case["kind"] == "one":
            sizes = [total]
        else:                                       # a few tensors hold most of it, as a model's matrices do
            share = torch.exp((1.0 if case["kind"] == "layer" else 2.0) * torch.randn(k, generator=torch.Generator().manual_seed(k))).double()
            sizes = [max(1, int(x)) for x in (share / share.sum() * total).tolist()]
        types = [DTYPES[case["dtype"]] if size > 2048 or case["kind"] != "model" else torch.float32 for size in sizes]
        s["grads"] = [(randn(size) * (1e-3 * 10 ** (i % 3))).to(t) for i, (size, t) in enumerate(zip(sizes, types))]
        # the results side by side in one buffer per type, each on a boundary of eight elements
        room = [-(-size // 8) * 8 for size in sizes]
        s["flat"] = {t: torch.zeros(sum(r for r, u in zip(room, types) if u == t), dtype=t, device="cuda") for t in dict.fromkeys(types)}
        at = dict.fromkeys(types, 0)
        s["out"] = []
        for size, r, t in zip(sizes, room, types):
            s["out"].append(s["flat"][t][at[t]:at[t] + size])
            at[t] += r
        s["max_norm"] = 1.0 if seed % 4 else 1e6    # now and then nothing is clipped
    return s


# ---- the plain forms ------------------------------------------------------------------------


def _plain_xent_loss(s):
    target = s["target"].long()
    live = (target >= 0) & (target < s["weight"].shape[0])
    z = s["hidden"].float() @ s["weight"].float().T
    top = z.amax(1, keepdim=True)
    lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]
    loss = lse - z.gather(1, target.clamp(0, z.shape[1] - 1)[:, None])[:, 0]
    return {"loss": torch.where(live, loss, 0.0), "lse": torch.where(live, lse, 0.0)}, z, live


def _plain_xent_step(s):
    outputs, z, live = _plain_xent_loss(s)
    g = torch.where(live, s["grad_loss"], 0.0)[:, None]
    grad = torch.exp(z - outputs["lse"][:, None])
    del z
    grad.scatter_add_(1, s["target"].long().clamp(0, grad.shape[1] - 1)[:, None], -torch.ones_like(g))
    grad = torch.where(live[:, None], grad * g, 0.0)
    outputs["grad_hidden"] = (grad @ s["weight"].float()).to(torch.bfloat16)
    outputs["grad_weight"] = (grad.T @ s["hidden"].float()).to(torch.bfloat16)
    return outputs


def _plain_parts(s):
    h, m = s["h"].float(), s["m"].float()
    gate = torch.ones((), device=h.device) if s["gate"] is None else s["gate"].float()
    gate = gate[:, None] if gate.dim() == 1 else gate
    if s["sigmoid"] and s["gate"] is not None:
        gate = 1 / (1 + torch.exp(-gate))
    a = 1 / torch.sqrt((m * m).mean(1, keepdim=True) + EPS)
    y = m * a * s["post_weight"].float()
    u = h + s["lam"] * gate * y
    return m, gate, a, y, u, 1 / torch.sqrt((u * u).mean(1, keepdim=True) + EPS)


def _plain_inject(s):
    _, _, _, _, u, b = _plain_parts(s)
    return {"out": u.to(s["h"].dtype), "normed": (u * b * s["next_weight"].float()).to(s["h"].dtype)}


def _plain_inject_grad(s):
    m, gate, a, y, u, b = _plain_parts(s)
    dn = s["grad_normed"].float()
    t = dn * s["next_weight"].float()
    du = s["grad_out"].float() + b * t - u * b ** 3 * (u * t).mean(1, keepdim=True)
    dy = s["lam"] * gate * du
    x = dy * s["post_weight"].float()
    dm = a * x - m * a ** 3 * (m * x).mean(1, keepdim=True)
    wt = s["next_weight"].dtype
    outputs = {"grad_h": du.to(s["h"].dtype), "grad_m": dm.to(s["h"].dtype), "grad_post": (dy * m * a).sum(0).to(wt), "grad_next": (dn * u * b).sum(0).to(wt)}
    if s["gate"] is not None:
        dg = s["lam"] * du * y
        if s["sigmoid"]:
            dg = dg * gate * (1 - gate)
        outputs["grad_gate"] = (dg if s["gate"].dim() == 2 else dg.sum(1)).to(s["gate"].dtype)
    return outputs


def _plain_clip(s):
    square = torch.stack([(x.float() * x.float()).sum(dtype=torch.float64) for x in s["grads"]])
    norm = torch.sqrt(square.sum())
    by = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    _ = [o.copy_(x.float() * by) for o, x in zip(s["out"], s["grads"])]
    return {"norm": norm.float(), "grads": list(s["flat"].values())}


def run(s):
    op = s["op"]
    if not own:
        if op == "xent_loss":
            return _plain_xent_loss(s)[0]
        return {"xent_step": _plain_xent_step, "inject": _plain_inject, "inject_grad": _plain_inject_grad, "clip": _plain_clip}[op](s)
    from paper_2607_07388_b200 import engine
    if op in ("xent_loss", "xent_step"):
        loss, lse = engine.xent_forward(s["hidden"], s["weight"], s["target"])
        if op == "xent_loss":
            return {"loss": loss, "lse": lse}
        grad_hidden, grad_weight = engine.xent_backward(s["grad_loss"], s["hidden"], s["weight"], s["target"], lse)
        return {"loss": loss, "lse": lse, "grad_hidden": grad_hidden, "grad_weight": grad_weight}
    if op == "inject":
        out, normed = engine.normed_inject_forward(s["h"], s["m"], s["post_weight"], s["next_weight"], s["gate"], sigmoid=s["sigmoid"], lam=s["lam"], eps=EPS)
        return {"out": out, "normed": normed}
    if op == "inject_grad":
        grads = engine.normed_inject_backward(s["grad_out"], s["grad_normed"], s["h"], s["m"], s["post_weight"], s["next_weight"], s["gate"],
                                              sigmoid=s["sigmoid"], lam=s["lam"], eps=EPS)
        names = ["grad_h", "grad_m", "grad_post", "grad_next", "grad_gate"]
        return {name: x for name, x in zip(names, grads) if x is not None}
    norm = engine.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
    return {"norm": norm, "grads": list(s["flat"].values())}


# ---- what a pass cannot do without ----------------------------------------------------------


def work(case):
    op = case["op"]
    if op in ("xent_loss", "xent_step"):
        n, v, d = case["rows"], case["vocab"], case["d"]
        live = max(1.0, n * (1 - case["ignored"]))
        once = 2 * (live + v) * d
        return {"bytes": int(once + 12 * n if op == "xent_loss" else 2 * once + 16 * n), "flops": int(2 * live * v * d * (1 if op == "xent_loss" else 3))}
    if op in ("inject", "inject_grad"):
        n, d, es = case["rows"], case["d"], SIZE[case["dtype"]]
        gate = {"none": 0, "scalar": 4 * n, "vector": n * d * es}[case["gate"]]
        weights = 2 * d * SIZE[case["weights"]]
        if op == "inject":
            return {"bytes": 4 * n * d * es + gate + weights, "flops": 10 * n * d}
        return {"bytes": 6 * n * d * es + 2 * gate + 2 * weights, "flops": 30 * n * d}
    return {"bytes": 2 * case["total"] * SIZE[case["dtype"]], "flops": 3 * case["total"]}


# ---- the definitions in 64 bits -------------------------------------------------------------


def _exact_xent(s, case):
    """A few rows at a time: log-softmax in 64 bits, and its derivative."""
    w, v = s["weight"].double(), case["vocab"]
    n, step = case["rows"], max(1, (1 << 27) // v)
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    gh = torch.zeros(s["hidden"].shape, dtype=torch.float64, device="cuda") if case["op"] == "xent_step" else None
    gw = None if gh is None else torch.zeros_like(w)
    rows = torch.nonzero((s["target"] >= 0) & (s["target"] < v))[:, 0]
    for at in rows.split(step):
        h, t = s["hidden"][at].double(), s["target"][at].long()
        z = h @ w.T
        norm = torch.logsumexp(z, 1)
        pick = torch.arange(len(at), device="cuda")
        loss[at], lse[at] = norm - z[pick, t], norm
        if gh is not None:
            p = z.sub_(norm[:, None]).exp_()
            p[pick, t] = torch.expm1(torch.log(p[pick, t]))
            p *= s["grad_loss"][at].double()[:, None]
            gh[at] = p @ w
            gw += p.T @ h
    outputs = {"loss": loss, "lse": lse}
    if gh is not None:
        outputs |= {"grad_hidden": gh, "grad_weight": gw}
    return outputs


def _exact_inject(s, case):
    """The derivatives by autograd in 64 bits from the forward formula, a slice of rows at a time."""
    grads = case["op"] == "inject_grad"
    wp, wn = (s[k].double().requires_grad_(grads) for k in ("post_weight", "next_weight"))
    found = {}
    for at in torch.arange(case["rows"], device="cuda").split(max(1, (1 << 25) // case["d"])):
        h, m = (s[k][at].double().requires_grad_(grads) for k in ("h", "m"))
        gate = None if s["gate"] is None else s["gate"][at].double().requires_grad_(grads)
        by = s["lam"]
        if gate is not None:
            x = gate if gate.dim() == 2 else gate.unsqueeze(1)
            by = by * (torch.sigmoid(x) if s["sigmoid"] else x)
        u = h + by * (wp * m / (m.square().mean(1, keepdim=True) + EPS).sqrt())
        normed = wn * u / (u.square().mean(1, keepdim=True) + EPS).sqrt()
        if grads:
            torch.autograd.backward([u, normed], [s["grad_out"][at].double(), s["grad_normed"][at].double()])
            part = {"grad_h": h.grad, "grad_m": m.grad} | ({} if gate is None else {"grad_gate": gate.grad})
        else:
            part = {"out": u, "normed": normed}
        for name, x in part.items():
            found.setdefault(name, []).append(x.detach())
    outputs = {name: torch.cat(x) for name, x in found.items()}
    return outputs | {"grad_post": wp.grad, "grad_next": wn.grad} if grads else outputs


def _exact_clip(s, case):
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(x.double())) ** 2 for x in s["grads"]))
    by = min(1.0, s["max_norm"] / norm)
    of = {t: [torch.nn.functional.pad(x.double() * by, (0, -len(x) % 8)) for x in s["grads"] if x.dtype == t] for t in s["flat"]}
    return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": [torch.cat(x) for x in of.values()]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("xent_loss", "xent_step"):
        return _exact_xent(s, case)
    return (_exact_clip if case["op"] == "clip" else _exact_inject)(s, case)
