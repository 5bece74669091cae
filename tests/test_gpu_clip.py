"""The norm of many gradients and clipping by it, against the formula in 64 bits."""
import math

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
    assert abs(float(norm) - want) <= 6 * 2.0 ** -24 * want, (float(norm), want)
    by = min(1.0, max_norm / want) if want > 0 and math.isfinite(want) else 1.0
    for x, y in zip(tensors, dev if out is None else out):
        y = y.cpu()
        if by == 1.0:
            assert torch.equal(x, y)
            continue
        e = x.double() * by
        half = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -24
        assert bool(((y.double() - e).abs() <= e.abs() * (half + 8 * 2.0 ** -24) + 1e-45).all())
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
