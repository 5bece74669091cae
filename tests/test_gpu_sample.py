"""Drawing tokens from logits against the definition in 64 bits: the same token for every row, and its probability."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def draw64(z, u, T=1.0, k=0, p=1.0, mp=0.0):
    """One row: (token, prob).  z float64; the settings are the fp32 values the library gets."""
    z = np.where(np.isnan(z), -np.inf, z)
    ids = np.flatnonzero(z > -np.inf)
    if not len(ids):
        return -1, 0.0
    top = z[ids].max()
    if not T > 0:
        return int(ids[np.argmax(z[ids])]), 1.0
    if mp > 0:
        ids = ids[z[ids] >= (top if mp >= 1 else top + T * math.log(mp))]
    ids = ids[np.argsort(-z[ids], kind="stable")]
    if k > 0:
        ids = ids[:k]
    with np.errstate(invalid="ignore"):
        w = np.where(z[ids] == top, 1.0, 0.0 if top == np.inf else np.exp((z[ids] - top) / T))      # +inf shares the draw
    if p < 1:
        run = np.cumsum(w)
        w = w[: int(np.searchsorted(run, max(p, 0.0) * run[-1], side="left")) + 1]
    run = np.cumsum(w)
    u = min(max(0.0 if math.isnan(u) else u, 0.0), 1 - 2.0 ** -24)
    at = int(np.searchsorted(run, u * run[-1], side="right"))
    return int(ids[at]), float(w[at] / run[-1])


def check(z, u, T=None, k=None, p=None, mp=None, out=None):
    """z: CPU tensor [B, V] of the type under test; the settings: fp32 / int32 numpy arrays or None."""
    from paper_2607_07388_b200 import engine
    dev = lambda a, dt: None if a is None else torch.from_numpy(np.asarray(a, dt)).to(DEV)
    token, prob = out or engine.sample_tokens(z.to(DEV), dev(u, np.float32), temperature=dev(T, np.float32), top_k=dev(k, np.int32),
                                              top_p=dev(p, np.float32), min_p=dev(mp, np.float32))
    token, prob = token.cpu().numpy(), prob.cpu().numpy()
    zn = z.double().numpy()
    f = lambda a, r, dflt: dflt if a is None else float(np.float32(a[r]))
    for r in range(len(zn)):
        e_token, e_prob = draw64(zn[r], f(u, r, 0), f(T, r, 1.0), int(f(k, r, 0)), f(p, r, 1.0), f(mp, r, 0.0))
        assert token[r] == e_token, (r, token[r], e_token)
        # weights exact to 1e-13, sums of integers in units of 2^-46 or finer against one: one rounding to fp32
        assert abs(prob[r] - e_prob) <= 2.0 ** -23 * e_prob + 1e-10, (r, prob[r], e_prob)
    return token, prob


def logits(seed, b, v, kind, spread=3.0, masked="none"):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.standard_normal((b, v)) * spread).astype(np.float32))
    if masked != "none":
        z[torch.from_numpy(rng.random((b, v)) < 0.4)] = float("-inf") if masked == "inf" else torch.finfo(TYPES[kind]).min
    return z.to(TYPES[kind]), rng


SETTINGS = {
    "plain": lambda g, b: {},
    "chat": lambda g, b: dict(T=g.choice([0.6, 0.8, 1.0], b), k=g.choice([1, 20, 50], b), p=g.choice([0.5, 0.9, 0.95], b)),
    "topp": lambda g, b: dict(p=g.choice([0.3, 0.9, 0.99, 0.9999], b)),
    "minp": lambda g, b: dict(mp=g.choice([0.0, 0.01, 0.1, 1.0], b), T=g.choice([0.5, 1.5], b)),
    "wide": lambda g, b: dict(k=g.choice([700, 2000, 30_000, 1 << 30], b), p=g.choice([0.7, 0.97, 1.0], b), T=g.choice([1.0, 2.0], b)),
    "all": lambda g, b: dict(T=g.choice([0.0, 0.1, 1.0, 5.0], b), k=g.choice([0, -3, 5, 5000], b), p=g.choice([1.0, 0.0, 0.8, 2.0], b),
                             mp=g.choice([0.0, 0.05, 1.0], b)),
}


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("settings", sorted(SETTINGS))
@pytest.mark.parametrize("b,v,spread,masked", [(5, 1, 1.0, "none"), (9, 7, 2.0, "none"), (16, 1000, 3.0, "inf"), (12, 4099, 0.3, "lowest"),
                                               (8, 33_001, 2.0, "none"), (6, 151_936, 1.0, "lowest"), (4, 262_143, 4.0, "inf")])
def test_against_definition(kind, settings, b, v, spread, masked):
    z, rng = logits(b * v, b, v, kind, spread, masked)
    check(z, rng.random(b).astype(np.float32), **SETTINGS[settings](rng, b))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("v", [64, 5000, 150_001])
def test_equal_logits(kind, v):
    """Rows of few distinct values, or of one: the order among equals is by index, and every sum is a whole number."""
    rng = np.random.default_rng(v)
    z = np.zeros((10, v), np.float32)
    z[1:4] = rng.integers(0, 2, (3, v))
    z[4] = -7.5
    z[5] = rng.integers(0, 3, v)
    z[6, v // 2] = 1.0
    z[7, : v // 2] = -0.0                                        # equal to +0
    z[8] = rng.integers(0, 2, v) * 1e-3
    z[9, ::2] = -60.0                                            # weights below any sum's unit
    z = torch.from_numpy(z).to(TYPES[kind])
    for u in (0.0, 0.25, 0.5, 0.999, 1 - 2.0 ** -24):
        check(z, np.full(10, u, np.float32))
    check(z, rng.random(10).astype(np.float32), k=np.full(10, v // 3), p=np.full(10, 0.5))
    check(z, rng.random(10).astype(np.float32), k=np.full(10, v - 1))
    check(z, rng.random(10).astype(np.float32), p=np.full(10, 0.75), T=np.full(10, 3.0))
    check(z, rng.random(10).astype(np.float32), T=np.full(10, np.inf))
    check(z, rng.random(10).astype(np.float32), T=np.full(10, 1e-30))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("v", [50, 40_000])
def test_rows_with_little_left(kind, v):
    rng = np.random.default_rng(v)
    z = (rng.standard_normal((10, v)) * 2).astype(np.float32)
    z[0] = -np.inf
    z[1] = np.nan
    z[2] = -np.inf; z[2, v - 1] = -5.0
    z[3, 3:] = np.nan
    z[4, 7] = np.inf
    z[5, [4, 9, v - 2]] = np.inf
    z[6] = torch.finfo(TYPES[kind]).min                          # nothing but the lowest value: equal logits
    z[7] = torch.finfo(TYPES[kind]).min; z[7, 11] = 0.0
    z[8, 5] = torch.finfo(TYPES[kind]).max
    z[9] *= 1e30
    z = torch.from_numpy(z).to(TYPES[kind])
    for settings in ({}, dict(T=np.zeros(10)), dict(k=np.full(10, 3), p=np.full(10, 0.6), mp=np.full(10, 0.2)), dict(T=np.full(10, np.inf)),
                     dict(T=np.full(10, 0.7), mp=np.full(10, 1.0))):
        token, prob = check(z, rng.random(10).astype(np.float32), **settings)
        assert token[0] == token[1] == -1 and prob[0] == prob[1] == 0


def test_parameters_outside_their_ranges():
    z, rng = logits(3, 12, 3000, "f32")
    n = np.nan
    u = np.array([0.3, -1.0, 1.0, 2.0, n, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5], np.float32)
    T = np.array([1, 1, 1, 1, 1, n, -1, 1e-45, 1e30, 1, 1, 1], np.float32)
    p = np.array([1, 1, 1, 0.9, 1, 1, 1, 1, 1, n, -1, 1], np.float32)
    mp = np.array([0, 0, 0, 0, 0, 0, 0, 0, 0, n, 0, 3], np.float32)
    k = np.array([-(1 << 31), (1 << 31) - 1, 0, 7, 1, 0, 0, 0, 0, 0, 0, 0], np.int32)
    check(z, u, T, k, p, mp)


def test_frequencies():
    """Evenly spread random numbers meet every token as often as its probability says."""
    v, n = 40, 20_000
    z, _ = logits(11, 1, v, "f32", 1.5)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    from paper_2607_07388_b200 import engine
    token, _ = engine.sample_tokens(z.expand(n, v).contiguous().to(DEV), torch.from_numpy(u).to(DEV))
    seen = np.bincount(token.cpu().numpy(), minlength=v)
    w = torch.softmax(z[0].double(), 0).numpy()
    assert np.abs(seen - n * w).max() <= 2          # each token owns one interval of u: off by at most one at both ends


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("v,ld,off", [(3001, 3003, 1), (3000, 3008, 0), (70_001, 70_011, 3), (5, 6, 1)])
def test_strided_rows(kind, v, ld, off):
    from paper_2607_07388_b200 import engine
    b = 5
    z, rng = logits(v, b, v, kind)
    store = torch.full((b * ld + off,), 50.0, dtype=TYPES[kind], device=DEV)      # what lies between the rows would win
    zs = torch.as_strided(store, (b, v), (ld, 1), off)
    zs.copy_(z)
    u = rng.random(b).astype(np.float32)
    p = np.full(b, 0.9, np.float32)
    check(z, u, p=p, out=engine.sample_tokens(zs, torch.from_numpy(u).to(DEV), top_p=torch.from_numpy(p).to(DEV)))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_vocabulary_beyond_shared_memory(kind):
    z, rng = logits(1, 2, 1_500_001, kind, 1.0)
    u = rng.random(2).astype(np.float32)
    check(z, u)
    check(z, u, p=np.array([0.9, 0.5]), k=np.array([0, 100_000]))


def test_rows_beyond_32_bit_offsets():
    from paper_2607_07388_b200 import engine
    v, b = 1 << 20, 4100
    z = torch.full((b, v), float("-inf"), dtype=torch.bfloat16, device=DEV)
    last, rng = logits(2, 1, v, "bf16", 1.0)
    z[-1] = last[0].to(DEV)
    u = torch.full((b,), 0.37, device=DEV)
    token, prob = engine.sample_tokens(z, u)
    assert (token[:-1] == -1).all()
    check(last, np.array([0.37], np.float32), out=(token[-1:], prob[-1:]))


def test_a_row_does_not_depend_on_its_batch():
    from paper_2607_07388_b200 import engine
    z, rng = logits(9, 40, 20_000, "bf16", 1.0)
    z, u = z.to(DEV), torch.from_numpy(rng.random(40).astype(np.float32)).to(DEV)
    p = torch.full((40,), 0.95, device=DEV)
    token, prob = engine.sample_tokens(z, u, top_p=p)
    again = engine.sample_tokens(z.flip(0), u.flip(0), top_p=p)
    assert torch.equal(token, again[0].flip(0)) and torch.equal(prob, again[1].flip(0))
    for r in (0, 17, 39):
        one = engine.sample_tokens(z[r:r + 1], u[r:r + 1], top_p=p[:1])
        assert one[0][0] == token[r] and one[1][0] == prob[r]


def test_captured_and_replayed_and_other_stream():
    from paper_2607_07388_b200 import engine
    z, rng = logits(4, 6, 50_000, "f32", 2.0)
    z, u = z.to(DEV), torch.from_numpy(rng.random(6).astype(np.float32)).to(DEV)
    k = torch.full((6,), 40, dtype=torch.int32, device=DEV)
    token, prob = engine.sample_tokens(z, u, top_k=k)
    zc, uc = torch.zeros_like(z), torch.zeros_like(u)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c_token, c_prob = engine.sample_tokens(zc, uc, top_k=k)
    for _ in range(2):
        zc.copy_(z); uc.copy_(u)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c_token, token) and torch.equal(c_prob, prob)
        zc.zero_(); uc.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert (c_token == 0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    one = engine.sample_tokens(z, u, top_k=k, stream=side)
    two = engine.sample_tokens(z, u.flip(0).contiguous(), top_k=k)          # at the same time on this one
    torch.cuda.synchronize()
    assert torch.equal(one[0], token) and two[0].shape == (6,)


def test_empty_batch_and_refusals():
    from paper_2607_07388_b200 import engine
    z, u = torch.zeros((3, 10), device=DEV), torch.zeros(3, device=DEV)
    token, prob = engine.sample_tokens(z[:0], u[:0])
    assert token.shape == prob.shape == (0,)
    for args, kw in (((z.double(), u), {}), ((z, u.double()), {}), ((z, u[:2]), {}), ((z, u.cpu()), {}), ((z.T.contiguous().T, u), {}),
                     ((z, u), dict(top_k=u)), ((z, u), dict(temperature=u[:1])), ((z, u), dict(top_p=0.9 * u.double()))):
        with pytest.raises(ValueError):
            engine.sample_tokens(*args, **kw)


@pytest.mark.parametrize("repeats", [300, 600, 1030])
def test_values_that_many_entries_share(repeats):
    """Every value held by 300, 600 or 1,030 entries: both searches' bins fit the list of 1,024 together, one after the other, or
    not at all."""
    rng = np.random.default_rng(repeats)
    v, b = 150_000 // repeats * repeats, 10
    values = np.linspace(-4, 4, v // repeats).astype(np.float32)
    z = torch.from_numpy(np.stack([rng.permutation(np.repeat(values, repeats)) for _ in range(b)]))
    u = rng.random(b).astype(np.float32)
    check(z, u, p=np.full(b, 0.9))
    check(z, u, p=np.full(b, 0.5), k=np.full(b, v // 2 + 17))
    check(z, u, k=np.full(b, 20_000), T=np.full(b, 2.0))


def bins_that_round_up():
    """A row whose estimated mass is 1.4e-5 too low.  With a least weight of exp(-32), 256 * 4,094 / 32 places make a unit of logit:
    nearly all entries lie half a place (0.51) beyond a whole one, and count as half a place further.  The last two filled bins
    hold 1,000 entries each, too many for one list."""
    unit = np.float32(256 * 4094 / 32)
    at = lambda place, n: np.full(n, -np.float32((place + 0.51) / unit), np.float32)
    body = [at(256 * b + 128, 1000) for b in (10, 11, 12, 13, 14)]
    total = sum(float(np.exp(x.astype(np.float64)).sum()) for x in body) + 1
    far = int(-math.log(total * 1.19e-5 / 1000) * float(unit)) // 256     # the bin in which 1,000 entries weigh 1.19e-5 of the row
    return np.concatenate([[np.float32(0)], *body, at(256 * (far - 1) + 128, 1000), at(256 * far + 128, 1000), [np.float32(-32)]]).astype(np.float32)


def test_an_estimate_that_ends_too_early():
    """The draw, searched for in a pass of its own from the exact mass, is to end behind all that the estimates say there is: the
    bins named for it are empty, and the row goes on by digits."""
    z = bins_that_round_up()
    unit = np.float32(256 * 4094 / 32)
    place = np.rint((-z * unit).astype(np.float32)).astype(np.int64)
    low = np.exp(-place.astype(np.float64) / float(unit)).sum() / np.exp(z.astype(np.float64)).sum()
    assert 1 - 1.53e-5 < low < 1 - 1.3e-5 and np.bincount(place >> 8).max() == 1000
    rng = np.random.default_rng(4)
    rows = 6
    zs = torch.from_numpy(np.stack([z] + [rng.permutation(z) for _ in range(rows - 1)]))
    u = np.array([1 - 2.0 ** -19, 1 - 2.0 ** -19, 1 - 2.0 ** -20, 1 - 2.0 ** -18, 1 - 2.0 ** -24, 0.5])
    check(zs, u, p=np.array([1 - 2.0 ** -20] * 5 + [0.99]))
    check(zs, u)
    check(zs, u, k=np.array([len(z) - 1] * rows), p=np.array([1 - 2.0 ** -20] * rows))


@pytest.mark.parametrize("v", [30, 5000, 300_000])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -100, 2.0 ** 60])
def test_bf16_values_of_every_size(v, scale):
    """Logits of any exponent beside each other, zeros of both signs and denormals among them: rows that are counted by value, and rows
    whose small logits do not fit the values counted."""
    rng = np.random.default_rng(v)
    b = 12
    z = rng.standard_normal((b, v)) * 3
    z[2:4] *= np.exp2(rng.integers(-40, 1, (2, v)))             # down to far below the 31 binades
    z[4:8] = np.where(rng.random((4, v)) < 0.6, rng.choice([0.0, -0.0], (4, v)), z[4:8])
    z[6, ::5] = 2.0 ** -130
    z[7, ::7] = -2.0 ** -133
    z[8] = -np.abs(z[8])
    z[9] = np.abs(z[9]) + 1
    z[10] = np.where(rng.random(v) < 0.5, 0.0, -2.0 ** -126)
    z[11] = np.where(rng.random(v) < 0.5, -0.0, -1e30)
    t = np.full(b, scale, np.float32)
    z = torch.from_numpy(z * np.where(z == 0, 1, scale)).to(torch.bfloat16)
    pick = lambda *choices: rng.choice(choices, b)
    check(z, rng.random(b), T=t)
    check(z, rng.random(b), T=t, p=pick(0.3, 0.9, 0.999))
    check(z, rng.random(b), T=t, k=pick(1, 7, v // 2, v - 1, v), p=pick(0.5, 1.0), mp=pick(0.0, 0.01, 1.0))
    check(z, np.where(np.arange(b) % 2, 0.0, 1 - 2.0 ** -24), T=t * 1e-3)


@pytest.mark.parametrize("v", [1100, 20_000, 262_144, 270_000, 1_100_000])
def test_bf16_draw_among_many_equals(v):
    """The drawn value held by more entries than the list: its entry is found by the digits of its index."""
    rng = np.random.default_rng(v)
    z = rng.choice([2.0, 1.0, -0.5], (4, v), p=[0.3, 0.6, 0.1]).astype(np.float32)
    z[1] = rng.choice([0.0, -0.0], v)
    z[2] = 3.0
    z[3, : v // 2] = -np.inf
    z = torch.from_numpy(z).to(torch.bfloat16)
    for u in (0.0, 0.37, 0.81, 1 - 2.0 ** -24):
        check(z, np.full(4, u))
        check(z, np.full(4, u), k=np.array([v // 2, v // 3, v - 1, v // 5]), p=np.array([0.7, 1.0, 0.9, 0.5]))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("top", [0.7, 5.0, 12.3, 1000.0, 5e4, 1e10, -5.0, -1e10])
@pytest.mark.parametrize("v", [700, 40_000])
def test_small_temperatures(kind, top, v):
    """Temperatures from those at which many logits weigh down to those at which one step below the maximum weighs nothing.  Three
    equal maxima, the logits one to eight steps below them, and the rest far away."""
    rng = np.random.default_rng(v)
    T = (np.abs(top) * 10.0 ** -np.arange(0.0, 24.0)).astype(np.float32)
    b = len(T)
    t = torch.tensor(top, dtype=torch.float32).to(TYPES[kind])
    near = [t]
    for _ in range(8):
        near.append(torch.nextafter(near[-1], torch.tensor(float("-inf"), dtype=TYPES[kind])))
    z = (float(t) - np.abs(rng.standard_normal((b, v))) * abs(top) * 1e-2).astype(np.float32)
    z = torch.from_numpy(z).to(TYPES[kind])
    z = torch.where(z >= t, near[8], z)
    at = rng.permutation(v)[:11]
    z[:, at[:3]] = t
    z[:, at[3:]] = torch.stack(near[1:])
    some = rng.permutation(v)[: v // 3]
    z[1::2, some] = torch.where(z[1::2, some] < near[8], torch.finfo(TYPES[kind]).min, z[1::2, some])       # every other row: masked ones too
    for u in (0.0, 0.5, 0.9, 0.999):
        check(z, np.full(b, u), T=T)
    check(z, rng.random(b), T=T, k=rng.choice([1, 2, 3, 5, v // 2], b), p=rng.choice([0.3, 0.9, 1.0], b))
    check(z, rng.random(b), T=T, p=np.full(b, 0.6), mp=rng.choice([0.0, 0.1, 1.0], b))
    check(z, rng.random(b), T=np.array([1e-30, 1e-38, 1e-45, 1e-9, 1e-10, 1e-11] * 4, np.float32))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("v", [50, 5000, 60_000])
def test_top_k_among_infinite_logits(kind, v):
    """Rows with two, three, a fifth of or nothing but +inf logits: top-k and top-p cut among them by index."""
    rng = np.random.default_rng(v)
    b = 8
    z = rng.standard_normal((b, v)).astype(np.float32)
    z[0, [v // 3, v - 2]] = np.inf
    z[1, [4, 9, v - 1]] = np.inf
    z[2, rng.permutation(v)[: v // 5]] = np.inf
    z[3] = np.inf
    z[4, [0, 1, 2]] = np.inf; z[4, 10:] = -np.inf; z[4, 5] = np.nan
    z[5, rng.permutation(v)[: v // 2]] = np.inf; z[5, ::7] = np.nan
    z[6, v // 2:] = np.inf
    z[7, 3] = np.inf
    z = torch.from_numpy(z).to(TYPES[kind])
    for u in (0.0, 0.4, 0.9, 1 - 2.0 ** -24):
        for k in (1, 2, 3, 7, max(8, v // 11), v // 3, v - 1):
            check(z, np.full(b, u), k=np.full(b, k))
            check(z, np.full(b, u), k=np.full(b, k), p=np.full(b, 0.7), T=np.full(b, 0.5))
    check(z, rng.random(b), k=np.full(b, 2), T=np.full(b, np.inf))
    check(z, rng.random(b), k=np.full(b, 2), mp=np.full(b, 0.3), T=np.full(b, 1e-12))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("b,v", [(2, 151_936), (6, 50_000), (70, 9001)])
def test_calls_at_the_same_time(kind, b, v):
    """Two streams draw from different rows by different numbers, over and over: each gets what it gets alone."""
    from paper_2607_07388_b200 import engine
    calls = []
    for i in range(2):
        z, rng = logits(17 * b + i, b, v, kind, 1.5)
        u = torch.from_numpy(rng.random(b).astype(np.float32)).to(DEV)
        p = torch.from_numpy(rng.choice([0.8, 0.95, 1.0], b).astype(np.float32)).to(DEV)
        calls.append((z.to(DEV), u, p))
    want = [engine.sample_tokens(z, u, top_p=p) for z, u, p in calls]
    assert not torch.equal(want[0][0], want[1][0])
    streams = [torch.cuda.Stream() for _ in calls]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(10):
        for i, (z, u, p) in enumerate(calls):
            got[i].append(engine.sample_tokens(z, u, top_p=p, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for token, prob in got[i]:
            assert torch.equal(token, want[i][0]) and torch.equal(prob, want[i][1])
