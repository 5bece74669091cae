"""The vocabulary product in 8 bits: conversion bit for bit, product against the formula in 64 bits, and the head on top."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

# the 127 non-negative finite values of e4m3, ascending: index = bit pattern
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def to_e4m3(x):
    """Bit patterns of the nearest e4m3 values of x (float32), ties to the even pattern, as uint8; NaN is 0x7F."""
    a = np.abs(x.astype(np.float64))
    hi = np.clip(np.searchsorted(E4M3, np.minimum(a, 448.0)), 1, 126)
    lo = hi - 1
    mid = (E4M3[lo] + E4M3[hi]) / 2
    up = (a > mid) | ((a == mid) & (hi % 2 == 0))
    bits = np.where(up, hi, lo).astype(np.uint8)
    bits[np.isnan(x)] = 0x7F
    return bits


def quantize64(x, block_rows):
    """(bit patterns without sign, sign, scale) by the definition; x float32 numpy."""
    r, c = x.shape
    kb = -(-c // 128)
    scale = np.zeros((-(-r // block_rows), kb), np.float32)
    y = np.zeros_like(x)
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(scale.shape[0]):
            for b in range(kb):
                at = np.s_[i * block_rows:(i + 1) * block_rows, 128 * b:128 * b + 128]
                big = np.abs(x[at]).max()                        # NaN propagates
                s = np.float32(big / np.float32(448))
                scale[i, b] = s if not np.isfinite(big) else max(s, np.float32(2.0 ** -126))
                y[at] = x[at] / scale[i, b]
    return to_e4m3(y), np.signbit(y), scale


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("r,c", [(1, 1), (3, 127), (5, 128), (128, 256), (130, 1000), (257, 1024), (40, 136), (9, 2051)])
def test_conversion(kind, block_rows, r, c):
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(r * c)
    x = (rng.standard_normal((r, c)) * np.exp2(rng.integers(-12, 12, (r, 1)))).astype(np.float32)
    x[0, : c // 2] = 0
    if r > 2:
        x[2] = rng.integers(-448, 449, c)                        # many exact values and ties
        x[2, c - 1] = 448
    xt = torch.from_numpy(x).to(TYPES[kind])
    q, scale = engine.quantize_fp8(xt.to(DEV), block_rows=block_rows)
    bits, sign, s = quantize64(xt.float().numpy(), block_rows)
    assert q.shape == (r, c) and np.array_equal(scale.cpu().numpy(), s)
    got = q.view(torch.uint8).cpu().numpy()
    assert np.array_equal(got & 0x7F, bits)
    assert np.array_equal((got >> 7).astype(bool)[bits > 0], sign[bits > 0])


@pytest.mark.parametrize("block_rows", [1, 128])
def test_conversion_of_extremes_and_strides(block_rows):
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(4)
    x = rng.standard_normal((260, 400)).astype(np.float32)
    x[0] = 0
    x[1, 130] = np.inf
    x[140, 5] = np.nan
    x[3] *= 1e-38; x[4] *= 1e-44; x[5] *= 3e38 / 5; x[131:, 256:] = 0
    store = torch.zeros((260, 407), device=DEV)
    for view in (store[:, :400], store[:, 3:403], torch.as_strided(store, (260, 400), (404, 1), 0)):
        view.copy_(torch.from_numpy(x))
        q, scale = engine.quantize_fp8(view, block_rows=block_rows)
        bits, _, s = quantize64(x, block_rows)
        assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)
        assert np.array_equal(q.view(torch.uint8).cpu().numpy() & 0x7F, bits)
        view.zero_()


def operands(seed, m, n, k):
    rng = np.random.default_rng(seed)
    pick = lambda r: torch.from_numpy((rng.standard_normal((r, k)) * 90).clip(-448, 448).astype(np.float32)).to(torch.float8_e4m3fn)
    kb = -(-k // 128)
    sa = torch.from_numpy(np.exp2(rng.uniform(-8, 2, (m, kb))).astype(np.float32))
    sw = torch.from_numpy(np.exp2(rng.uniform(-8, 2, (-(-n // 128), kb))).astype(np.float32))
    return pick(m), sa, pick(n), sw


def padded(t):
    """The rows of an e4m3 matrix on the device, starting on 16-byte boundaries."""
    r, k = t.shape
    store = torch.zeros((r, -(-k // 16) * 16), dtype=torch.uint8, device=DEV)
    store[:, :k] = t.view(torch.uint8).to(DEV)
    return store.view(torch.float8_e4m3fn)[:, :k]


def product64(a, sa, w, sw):
    """The formula, and the sum of the magnitudes of its terms."""
    k, n = a.shape[1], w.shape[0]
    a64 = a.to(DEV).double() * sa.to(DEV).double().repeat_interleave(128, 1)[:, :k]
    w64 = w.to(DEV).double() * sw.to(DEV).double().repeat_interleave(128, 1)[:, :k].repeat_interleave(128, 0)[:n]
    return a64 @ w64.T, a64.abs() @ w64.abs().T


def check_product(out, a, sa, w, sw, kind):
    want, size = product64(a, sa, w, sw)
    kb = sa.shape[1]
    # within a block 128 exact products are added, each addition cutting at most one unit of 2^-23 of the running sum; then the
    # product of the scales, its product with the sum and the addition over blocks, half a unit each
    tol = size * (132 * 2.0 ** -23 + (kb + 2) * 2.0 ** -24) + want.abs() * (2.0 ** -8 if kind == "bf16" else 2.0 ** -24) + 1e-37
    bad = (out.double() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float(((out.double() - want).abs() / tol).max()))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 8, 16), (3, 129, 128), (16, 1000, 144), (17, 128, 1024), (32, 5000, 130), (33, 300, 4096),
                                   (64, 20_003, 256), (65, 148 * 128 + 1, 384), (128, 777, 2050), (129, 4099, 272), (200, 1187, 1024),
                                   (256, 19_000, 128), (257, 130, 512), (600, 1111, 640), (1000, 2500, 1024), (1, 60, 8200)])
def test_product(kind, m, n, k):
    from paper_2607_07388_b200 import binding as tfe
    from paper_2607_07388_b200 import engine
    a, sa, w, sw = operands(m + n + k, m, n, k)
    out = engine.matmul_fp8(padded(a), sa.to(DEV), padded(w), sw.to(DEV), out_dtype=TYPES[kind])
    assert tfe.tfe_matmul_fp8_status() == 0
    check_product(out, a, sa, w, sw, kind)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_product_of_whole_numbers_is_exact(m):
    """Small integers: every partial sum is exact in fp32, in any order."""
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(m)
    n, k = 2003, 1024
    ai, wi = rng.integers(-8, 9, (m, k)), rng.integers(-8, 9, (n, k))
    a, w = (torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).to(DEV) for x in (ai, wi))
    sa = torch.from_numpy(np.exp2(rng.integers(0, 3, (m, 8))).astype(np.float32)).to(DEV)
    sw = torch.from_numpy(np.exp2(rng.integers(0, 3, (16, 8))).astype(np.float32)).to(DEV)
    out = engine.matmul_fp8(a, sa, w, sw)
    want, _ = product64(a, sa, w, sw)
    assert torch.equal(out.double(), want)


@pytest.mark.parametrize("m", [2, 300])
def test_product_into_strided_output(m):
    from paper_2607_07388_b200 import engine
    a, sa, w, sw = operands(m, m, 1003, 256)
    store = torch.full((m, 1011), 5.0, device=DEV)
    out = store[:, 3:1006]
    got = engine.matmul_fp8(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), out=out)
    assert got.data_ptr() == out.data_ptr()
    check_product(out, a, sa, w, sw, "f32")
    assert torch.equal(out, engine.matmul_fp8(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV)))
    out.fill_(5.0)
    assert (store == 5.0).all()


@pytest.mark.parametrize("m", [3, 300])
def test_not_a_number_stays_in_its_row_and_column(m):
    from paper_2607_07388_b200 import engine
    a, sa, w, sw = operands(m, m, 500, 256)
    a8, w8 = a.view(torch.uint8).clone(), w.view(torch.uint8).clone()
    a8[1, 7] = 0x7F
    w8[130, 200] = 0xFF
    sw[3, 1] = float("inf")                                      # rows 384..499
    out = engine.matmul_fp8(a8.view(torch.float8_e4m3fn).to(DEV), sa.to(DEV), w8.view(torch.float8_e4m3fn).to(DEV), sw.to(DEV))
    nan = torch.isnan(out)
    assert nan[1, :384].all() and nan[:, 130].all()
    assert not torch.isfinite(out[:, 384:]).any()
    nan[1] = False; nan[:, 130] = False
    assert not nan[:, :384].any()


def test_head_in_8_bits():
    """Logits, sampling and the top entries against the same weights and states in 64 bits."""
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(8)
    V, d, B = 9001, 256, 5
    w = torch.from_numpy((rng.standard_normal((V, d)) * 0.1).astype(np.float32)).to(torch.bfloat16).to(DEV)
    h = torch.from_numpy(rng.standard_normal((B, d)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    head = engine.QuantizedHead(w)
    z = head.logits(h)
    want = h.double() @ w.double().T
    # each factor is off by half a step of e4m3 at most, 2^-4 of its value (or of its block's smallest normal)
    size = h.double().abs() @ w.double().abs().T
    small = (h.double().abs().amax() * w.double().abs().sum(1) + w.double().abs().amax() * h.double().abs().sum(1)[:, None]) * 2.0 ** -10 / 448 * 2
    assert ((z.double() - want).abs() <= size * (2.0 ** -3 + 2.0 ** -8) + small).all()
    assert (torch.linalg.norm(z.double() - want) / torch.linalg.norm(want)).item() < 2.0 ** -4
    u = torch.from_numpy(rng.random(B).astype(np.float32)).to(DEV)
    token, prob = head.sample(h, u, top_k=torch.full((B,), 20, dtype=torch.int32, device=DEV))
    t2, p2 = engine.sample_tokens(z, u, top_k=torch.full((B,), 20, dtype=torch.int32, device=DEV))
    assert torch.equal(token, t2) and torch.equal(prob, p2)


def test_captured_and_replayed_and_other_stream():
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(2)
    w = torch.from_numpy(rng.standard_normal((5000, 128)).astype(np.float32)).to(DEV)
    h = torch.from_numpy(rng.standard_normal((300, 128)).astype(np.float32)).to(DEV)
    head = engine.QuantizedHead(w)
    z = head.logits(h)
    hc = torch.zeros_like(h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zc = head.logits(hc)
    for _ in range(2):
        hc.copy_(h)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(zc, z)
        hc.zero_()
        graph.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    one, two = head.logits(h, stream=side), head.logits(h.flip(0))       # at the same time
    torch.cuda.synchronize()
    assert torch.equal(one, z) and torch.equal(two.flip(0), z)


def test_empty_batch_and_refusals():
    from paper_2607_07388_b200 import engine
    a, sa, w, sw = (x.to(DEV) for x in operands(1, 4, 200, 256))
    assert engine.matmul_fp8(a[:0], sa[:0], w, sw).shape == (0, 200)
    q, s = engine.quantize_fp8(torch.empty((0, 64), device=DEV))
    assert q.shape == (0, 64) and s.shape == (0, 1)
    for args in ((a.float(), sa, w, sw), (a, sa[:3], w, sw), (a, sa, w, sw[:1]), (a, sa.double(), w, sw), (a, sa, w[:, :128], sw[:, :1]),
                 (a.cpu(), sa, w, sw), (a, sa, w[:0], sw[:0])):
        with pytest.raises(ValueError):
            engine.matmul_fp8(*args)
    odd = torch.zeros((4, 250), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    with pytest.raises(ValueError):                              # rows off 16-byte boundaries
        engine.matmul_fp8(odd, sa, w[:, :250], sw)
    with pytest.raises(ValueError):
        engine.matmul_fp8(a, sa, w, sw, out_dtype=torch.float16)
    with pytest.raises(ValueError):
        engine.matmul_fp8(a, sa, w, sw, out=torch.empty((4, 201), device=DEV))
    for bad in (0, 2, 64):
        with pytest.raises(ValueError):
            engine.quantize_fp8(torch.zeros((4, 64), device=DEV), block_rows=bad)
    with pytest.raises(ValueError):
        engine.quantize_fp8(torch.zeros((4, 64), dtype=torch.float16, device=DEV))
    with pytest.raises(ValueError):
        engine.QuantizedHead(torch.zeros((4, 72), device=DEV))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_conversion_next_to_the_rounding_borders(kind):
    """Values whose quotients lie on the borders between e4m3 values and next to them, for many scales: half a million
    quotients bit for bit, of scales over the whole range."""
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(77)
    r = 4096
    x = np.zeros((r, 128), np.float32)
    big = np.exp2(rng.uniform(-120, 120, r)).astype(np.float32)
    border = (E4M3[:-1] + E4M3[1:]) / 2
    for i in range(r):
        s = np.float32(big[i] / np.float32(448))
        x[i, 1:] = (rng.choice(border, 127) * np.float64(s)).astype(np.float32)
        x[i, 1:] = (x[i, 1:].view(np.int32) + rng.integers(-2, 3, 127).astype(np.int32)).view(np.float32)
        x[i, 0] = big[i]
    xt = torch.from_numpy(x).to(TYPES[kind])
    q, scale = engine.quantize_fp8(xt.to(DEV))
    bits, _, s = quantize64(xt.float().numpy(), 1)
    assert np.array_equal(scale.cpu().numpy(), s)
    assert np.array_equal(q.view(torch.uint8).cpu().numpy() & 0x7F, bits)


def test_output_on_its_operands_is_refused():
    """`out` over the bytes of an operand: refused.  Beside it in the same storage: taken."""
    from paper_2607_07388_b200 import engine
    a, sa, w, sw = (x.to(DEV) for x in operands(2, 4, 128, 256))
    room = torch.zeros(4 * 256 + 4 * 128 * 4, dtype=torch.uint8, device=DEV)
    inside = room[: 4 * 256].view(4, 256).view(torch.float8_e4m3fn)
    inside.copy_(a)
    at = lambda first: room[first: first + 4 * 128 * 2].view(torch.bfloat16).view(4, 128)
    for first in (0, 1008):
        with pytest.raises(ValueError):
            engine.matmul_fp8(inside, sa, w, sw, out=at(first))
    over_w = w.reshape(-1).view(torch.uint8)[-1024:].view(torch.bfloat16).view(4, 128)
    with pytest.raises(ValueError):
        engine.matmul_fp8(a, sa, w, sw, out=over_w)
    want = engine.matmul_fp8(a, sa, w, sw, out_dtype=torch.bfloat16)
    assert torch.equal(engine.matmul_fp8(inside, sa, w, sw, out=at(1024)), want)


def test_conversion_of_more_groups_than_32_bits_of_threads():
    """2^28 groups are 2^32 threads: the rows beyond are converted like the first."""
    from paper_2607_07388_b200 import engine
    r = (1 << 28) + 1000
    x = torch.full((r, 1), 3.0, dtype=torch.bfloat16, device=DEV)
    ends = [(0, 1000), ((1 << 28) - 500, (1 << 28) + 500), (r - 1000, r)]
    rng = np.random.default_rng(28)
    given = [torch.from_numpy(rng.standard_normal((b - a, 1)).astype(np.float32)).to(torch.bfloat16) for a, b in ends]
    for (a, b), part in zip(ends, given):
        x[a:b] = part.to(DEV)
    q, scale = engine.quantize_fp8(x)
    for a, b in ends:
        bits, sign, s = quantize64(x[a:b].float().cpu().numpy(), 1)
        assert np.array_equal(scale[a:b].cpu().numpy(), s)
        got = q[a:b].view(torch.uint8).cpu().numpy()
        assert np.array_equal(got & 0x7F, bits) and np.array_equal(got >> 7, sign)
    assert int((scale == np.float32(3) / np.float32(448)).sum()) >= r - 3000


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(3, 1003, 640), (40, 30_001, 256), (64, 77, 128), (300, 1003, 640), (65, 90_001, 128)])
def test_waits_that_run_out(m, n, k, kind):
    """Every wait of the kernel counts as run out: all results are NaN, nothing beside them is touched, the status tells once, and the
    next product is right again."""
    from paper_2607_07388_b200 import binding as tfe
    from paper_2607_07388_b200 import engine
    a, sa, w, sw = operands(m + n, m, n, k)
    args = (a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV))
    store = torch.full((m, n + 8), 5.0, dtype=TYPES[kind], device=DEV)
    out = store[:, 3:n + 3]
    assert engine.matmul_fp8_status() == 0
    tfe.tfe_matmul_fp8_give_up(True)
    try:
        engine.matmul_fp8(*args, out=out)
        torch.cuda.synchronize()
    finally:
        tfe.tfe_matmul_fp8_give_up(False)
    assert torch.isnan(out).all()
    token, prob = engine.sample_tokens(out, torch.full((m,), 0.5, device=DEV))
    assert (token == -1).all() and (prob == 0).all()
    good = engine.matmul_fp8(*args, out_dtype=TYPES[kind])
    assert engine.matmul_fp8_status() != 0                       # of the call before: the good one has set nothing
    assert engine.matmul_fp8_status() == 0
    check_product(good, a, sa, w, sw, kind)
    head = engine.QuantizedHead(torch.ones((16, 16), device=DEV))
    assert head.status() == 0
    out.fill_(5.0)
    assert (store == 5.0).all()


@pytest.mark.parametrize("which", [1, 3])
def test_output_on_the_scales_is_refused(which):
    from paper_2607_07388_b200 import engine
    args = [x.to(DEV) for x in operands(5, 3, 100, 1024)]
    want = engine.matmul_fp8(*args)
    size = args[which].numel()
    room = torch.zeros(size + 300, device=DEV)
    held = room[:size].view(args[which].shape)
    held.copy_(args[which])
    args[which] = held
    for first in (0, size - 1):
        with pytest.raises(ValueError):
            engine.matmul_fp8(*args, out=room[first: first + 300].view(3, 100))
    assert torch.equal(engine.matmul_fp8(*args, out=room[size: size + 300].view(3, 100)), want)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (3, 200, 8), (40, 129, 1000), (70, 300, 100), (130, 257, 2051)])
def test_converted_matrices_of_any_width_are_operands(m, n, k, kind):
    """What quantize_fp8 gives goes into matmul_fp8 as it is, whatever the width."""
    from paper_2607_07388_b200 import engine
    rng = np.random.default_rng(m + n + k)
    x, w = (torch.from_numpy(rng.standard_normal((r, k)).astype(np.float32)).to(TYPES[kind]).to(DEV) for r in (m, n))
    (q, sa), (qw, sw) = engine.quantize_fp8(x), engine.quantize_fp8(w, 128)
    for t, src, rows in ((q, x, 1), (qw, w, 128)):
        assert t.shape == src.shape
        bits, sign, _ = quantize64(src.float().cpu().numpy(), rows)
        got = t.view(torch.uint8).cpu().numpy()
        assert np.array_equal(got & 0x7F, bits) and np.array_equal((got >> 7).astype(bool)[bits > 0], sign[bits > 0])
    check_product(engine.matmul_fp8(q, sa, qw, sw), q, sa, qw, sw, "f32")


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("c,ldq,off", [(100, 100, 0), (100, 112, 0), (1000, 1008, 0), (1000, 1003, 0), (64, 70, 5), (136, 144, 8)])
def test_conversion_into_rows_apart(c, ldq, off, block_rows):
    """Rows of q at any distance; what lies between them is not touched."""
    from paper_2607_07388_b200 import binding as tfe
    from paper_2607_07388_b200 import engine
    r = 131
    x = torch.randn((r, c), generator=torch.Generator().manual_seed(c)).to(DEV)
    want, want_scale = engine.quantize_fp8(x, block_rows)
    store = torch.full((off + r * ldq,), 0x55, dtype=torch.uint8, device=DEV)
    q = torch.as_strided(store, (r, c), (ldq, 1), off)
    scale = torch.empty_like(want_scale)
    tfe.tfe_quantize_fp8_ld(x.data_ptr(), tfe.DTYPE_F32, r, c, c, block_rows, q.data_ptr(), ldq, scale.data_ptr())
    assert torch.equal(q, want.view(torch.uint8)) and torch.equal(scale, want_scale)
    q.fill_(0x55)
    assert (store == 0x55).all()
    dense = torch.empty((r, c), dtype=torch.uint8, device=DEV)
    tfe.tfe_quantize_fp8(x.data_ptr(), tfe.DTYPE_F32, r, c, c, block_rows, dense.data_ptr(), scale.data_ptr())
    assert torch.equal(dense, want.view(torch.uint8))
