"""The norm of many gradients and clipping by it, against the formula in 64 bits."""
import math
import os
import random

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def make(seed, sizes, types, scale=1.0):
    rng = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=rng) * scale).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def reference(tensors):
    return math.sqrt(math.fsum(float((x.double() ** 2).sum()) for x in tensors))


def check(tensors, max_norm, out=None, dev=None):
    """The norm: sums of 4 or 8 squares in fp32 (at most 8 half-steps of 2^-24 relative, halved by the root), the rest in fp64, one
    rounding.  A result: the factor's rounding, the product's, and the type's."""
    from paper_2607_07388_b200 import engine
    dev = [x.to(DEV) for x in tensors] if dev is None else dev
    want = reference(tensors)
    norm = engine.clip_grad_norm(dev, max_norm, out=out)
    assert norm.shape == () and norm.dtype == torch.float32
    if want >= 2.0 ** 128 * (1 - 2.0 ** -25):       # nearer to 2^128 than to fp32's greatest number 2^128 (1 - 2^-24): no fp32 number but inf
        assert float(norm) == math.inf
        want = math.inf
    else:
        assert abs(float(norm) - want) <= 6 * 2.0 ** -24 * want, (float(norm), want)
    by = min(1.0, max_norm / want) if want > 0 and math.isfinite(want) else 1.0
    for x, y in zip(tensors, dev if out is None else out):
        y = y.cpu()
        if by == 1.0:
            assert torch.equal(x, y)
            continue
        e = x.double() * by
        # below 2^-126 the numbers of a type with p bits of fraction lie 2^(-126 - p) apart (bf16: 7, fp32: 23), half of which is a rounding
        half, least = (2.0 ** -8, 2.0 ** -134) if x.dtype == torch.bfloat16 else (2.0 ** -24, 2.0 ** -150)
        assert bool(((y.double() - e).abs() <= e.abs() * (half + 8 * 2.0 ** -24) + least).all())
    return norm


@pytest.mark.parametrize("sizes", [[1], [7], [0, 3, 0], [8192], [8193], [100_003], [5, 8192, 1, 70_001, 0, 16], [64] * 65, [300] * 900, [17] * 901, [3] * 2000, [3_000_001, 2]])
@pytest.mark.parametrize("types", [[torch.bfloat16], [torch.float32], [torch.bfloat16, torch.float32]])
def test_sizes(sizes, types):
    x = make(len(sizes), sizes, types)
    norm = reference(x)
    check(x, 0.37 * norm)
    check(x, 2.0 * norm)
    check(x, 0.37 * norm, out=[torch.empty_like(t, device=DEV) for t in x])
    check(x, 2.0 * norm, out=[torch.empty_like(t, device=DEV) for t in x])


def test_elements_beyond_the_range_of_their_squares():
    """Squares that leave fp32 on either side, in vectors of their own and mixed."""
    for scale in (1e25, 1e-25, 3e37):
        x = make(1, [1000, 37], [torch.float32], scale)
        check(x, 0.5 * reference(x))
    x = [torch.tensor([1e30, 1e-30, 0.0, 2.0] * 50), torch.tensor([3e38, 1e-38]).bfloat16(), torch.zeros(4000)]
    check(x, 0.25 * reference(x))
    from paper_2607_07388_b200 import engine
    assert float(engine.grad_norm(torch.zeros(5000, device=DEV))) == 0.0
    check([torch.zeros(5000)], 0.0)
    tiny = torch.full((5000,), 1e-40)                           # below the normal numbers
    assert abs(float(engine.grad_norm(tiny.to(DEV))) - reference([tiny])) <= 1e-44


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("at", [0, 4999])
def test_norms_that_are_not_finite_leave_the_elements(value, at):
    from paper_2607_07388_b200 import engine
    x = make(2, [5000, 100], [torch.float32, torch.bfloat16])
    x[0][at] = value
    dev = [t.to(DEV) for t in x]
    norm = engine.clip_grad_norm(dev, 1.0)
    assert not torch.isfinite(norm) and torch.isnan(norm) == (value != value)
    for a, b in zip(x, dev):
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b.cpu()))
    out = [torch.zeros_like(t) for t in dev]
    engine.clip_grad_norm(dev, 1.0, out=out)
    for a, b in zip(x, out):
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b.cpu()))


def test_limits():
    x = make(3, [3000], [torch.bfloat16])
    check(x, float("inf"))
    check(x, 0.0)
    n = reference(x)
    check(x, n * 1.001)
    check(x, n * 0.999)
    from paper_2607_07388_b200 import engine
    assert abs(float(engine.grad_norm([t.to(DEV) for t in x])) - n) <= 6 * 2.0 ** -24 * n
    assert abs(float(engine.grad_norm(x[0].to(DEV))) - n) <= 6 * 2.0 ** -24 * n


def test_views_of_one_buffer():
    """Tensors side by side at odd places, and results at others: what lies between stays."""
    from paper_2607_07388_b200 import engine
    for t in (torch.bfloat16, torch.float32):
        flat, room = torch.randn(40_000).to(t), torch.full((40_100,), 7.0).to(t).to(DEV)
        cuts = [1, 4, 4099, 4100, 30_001, 39_999]
        cpu = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
        dev = flat.to(DEV)
        views = [dev[a:b] for a, b in zip(cuts, cuts[1:])]
        out = [room[a + 3 * i:b + 3 * i] for i, (a, b) in enumerate(zip(cuts, cuts[1:]))]
        check(cpu, 0.1 * reference(cpu), out=out, dev=views)
        assert torch.equal(dev.cpu(), flat)
        covered = torch.zeros(40_100, dtype=torch.bool)
        for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
            covered[a + 3 * i:b + 3 * i] = True
        assert bool((room.cpu()[~covered] == 7.0).all())
        check(cpu, 0.1 * reference(cpu), dev=views)
        assert torch.equal(dev.cpu()[:1], flat[:1]) and torch.equal(dev.cpu()[39_999:], flat[39_999:])


def test_some_results_in_place():
    x = make(4, [500, 9000, 3], [torch.float32, torch.bfloat16])
    dev = [t.to(DEV) for t in x]
    out = [dev[0], torch.empty_like(dev[1]), dev[2]]
    version = dev[0]._version
    check(x, 0.5 * reference(x), out=out, dev=dev)
    assert torch.equal(dev[1].cpu(), x[1]) and dev[0]._version > version


def test_more_elements_than_32_bits_count():
    from paper_2607_07388_b200 import engine
    n = 2 ** 31 + 4097
    x = torch.full((n,), 0.5, dtype=torch.bfloat16, device=DEV)
    x[-1] = 64.0
    norm = float(engine.clip_grad_norm(x, 1.0))
    want = math.sqrt((n - 1) * 0.25 + 4096.0)
    assert abs(norm - want) <= 1e-6 * want
    by = 1.0 / want
    assert abs(float(x[0]) - 0.5 * by) <= 0.5 * by * 2.0 ** -7 and abs(float(x[-1]) - 64 * by) <= 64 * by * 2.0 ** -7 and torch.equal(x[:5], x[-6:-1])


def test_captured_and_two_streams():
    from paper_2607_07388_b200 import engine
    data = [make(s, [70_000, 33, 8000] * 30, [torch.bfloat16, torch.float32]) for s in (5, 6)]
    dev = [[t.to(DEV) for t in x] for x in data]
    streams = [torch.cuda.Stream() for _ in dev]
    torch.cuda.synchronize()
    outs = [[[torch.empty_like(t) for t in x] for _ in range(3)] for x in dev]
    torch.cuda.synchronize()
    norms = [[engine.clip_grad_norm(x, 1.0, out=o, stream=s) for o in oo] for x, oo, s in zip(dev, outs, streams)]
    torch.cuda.synchronize()
    for x, oo, nn in zip(data, outs, norms):
        for o, n in zip(oo, nn):
            assert abs(float(n) - reference(x)) <= 6 * 2.0 ** -24 * reference(x)
            assert all(torch.equal(a, b) for a, b in zip(o, oo[0]))
    held = [t.clone() for t in dev[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = engine.clip_grad_norm(held, 1.0)
    for k in (1, 0):
        for a, b in zip(held, dev[k]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, norms[k][0]) and all(torch.equal(a, b) for a, b in zip(held, outs[k][0]))


def test_refusals():
    from paper_2607_07388_b200 import engine
    from paper_2607_07388_b200.binding import TfeError
    x = torch.ones(100, device=DEV)
    for call in (lambda: engine.clip_grad_norm([], 1.0), lambda: engine.clip_grad_norm([x.double()], 1.0), lambda: engine.clip_grad_norm([x.cpu()], 1.0),
                 lambda: engine.clip_grad_norm([x, x.cpu()], 1.0), lambda: engine.clip_grad_norm([x[::2]], 1.0), lambda: engine.clip_grad_norm(x, -1.0),
                 lambda: engine.clip_grad_norm(x, float("nan")), lambda: engine.clip_grad_norm([x], 1.0, out=[x[:99]]), lambda: engine.clip_grad_norm([x], 1.0, out=[x, x]),
                 lambda: engine.clip_grad_norm([x], 1.0, out=[x.bfloat16()]), lambda: engine.grad_norm([x.half()])):
        with pytest.raises(ValueError):
            call()
    y = torch.ones(200, device=DEV)
    for call in (lambda: engine.clip_grad_norm([x, x], 1.0), lambda: engine.clip_grad_norm([y[:150], y[100:]], 1.0), lambda: engine.clip_grad_norm([y[:100], y[100:]], 1.0, out=[y[100:], x]),
                 lambda: engine.clip_grad_norm([y[:100]], 1.0, out=[y[50:150]]), lambda: engine.clip_grad_norm([x, y[:100]], 1.0, out=[y[100:], y[100:]])):
        with pytest.raises(TfeError):
            call()
    assert float(engine.grad_norm([x, x])) == pytest.approx(200 ** 0.5, rel=1e-6)       # nothing is written: the same tensor may count twice
    assert torch.equal(x, torch.ones(100, device=DEV)) and torch.equal(y, torch.ones(200, device=DEV))


@pytest.mark.parametrize("seed", range(int(os.environ.get("TFE_RANDOM_CASES", "12"))))
def test_random_sizes(seed):
    rng = random.Random(3000 + seed)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    sizes = [rng.choice([0, 1, log(1, 200_000)]) for _ in range(log(1, 1200))] + [log(1, 300_000)]
    x = make(seed, sizes, rng.choice([[torch.bfloat16], [torch.float32], [torch.bfloat16, torch.float32, torch.float32]]), rng.choice([1.0, 1e-6, 1e4]))
    flat = {t: torch.cat([y for y in x if y.dtype == t] + [torch.zeros(0, dtype=t)]).to(DEV) for t in (torch.bfloat16, torch.float32)}
    at, dev = {torch.bfloat16: 0, torch.float32: 0}, []
    for y in x:                         # side by side, at whatever boundary
        dev.append(flat[y.dtype][at[y.dtype]:at[y.dtype] + y.numel()])
        at[y.dtype] += y.numel()
    out = None if rng.random() < 0.5 else [torch.empty_like(y) for y in dev]
    norm = reference(x)
    check(x, norm * rng.choice([0.3, 0.9, 1.5]) if norm > 0 else 1.0, out=out, dev=dev)


def test_inference_tensors_and_parameters():
    """Tensors that have no version among others that have one; parameters, and a generator instead of a list."""
    from paper_2607_07388_b200 import engine
    with torch.inference_mode():
        a = torch.ones(300, device=DEV)
    b, p = torch.ones(500, device=DEV), torch.nn.Parameter(torch.ones(10, 20, device=DEV).bfloat16())
    version = b._version
    with torch.no_grad():
        norm = engine.clip_grad_norm((x for x in (a, b, p)), 1.0)
    assert abs(float(norm) - 1000 ** 0.5) <= 1e-4 and b._version > version
    assert abs(float(engine.grad_norm([a, b, p])) - 1.0) <= 2.0 ** -8
