"""Unbiased rounding of 8-bit AdamW states: its draws, its mean, and runs of thousands of steps against 32-bit states.

The definition (gnnhot.h) fixes every operation, so the kernel's codes and scales have to be equal to numpy's.  Long runs are compared
by the spread that the definition leaves: the variance that a step adds to a second moment of code c is that of a rounding between values 4 / c
of it apart, (1 - beta2) v * 4 v / c at most, and a step takes 2 (1 - beta2) of the variance back, so its relative spread is sqrt(2 / c)."""
import numpy as np
import pytest
import torch

import paper_2311_06837_amd as P
from paper_2311_06837_amd import binding as B

f32, u64 = np.float32, np.uint64
B1, B2 = 0.9, 0.999
MASK = u64(0xffffffff)
C0, C1, C2 = u64(0x9E3779B9), u64(0xBB67AE85), u64(0x6A09E667)


# ---- the definition ----------------------------------------------------------------------------------------------
def fold(x, c):
    p = (np.asarray(x, u64) & MASK) * c
    return (p ^ (p >> u64(32))) & MASK


def draws(seed, step, tensor, i):
    """The 32 bits of elements i."""
    i = np.asarray(i, u64)
    s = fold(u64(seed) + C0, C1)
    s = fold(s ^ u64(step & 0xffffffff), C2)
    s = fold(s + u64(step >> 32) + C0, C1)
    k0 = fold(s ^ u64(tensor), C2)
    k1 = fold(k0 + C0, C1)
    high = i >> u64(32)
    return fold(fold((i & MASK) ^ ((k0 + high * C2) & MASK), C0) ^ ((k1 + high * C0) & MASK), C1)


def reversed_bits(x):
    b = np.ascontiguousarray(x.astype(">u4")).view(np.uint8)
    return np.packbits(np.unpackbits(b).reshape(-1, 32)[:, ::-1], axis=1).view(">u4").ravel().astype(u64)


def unit(x):
    return (((x >> u64(9)).astype(np.float64) + 0.5) * 2.0 ** -23).astype(f32)


def values(steps):
    """Values of the codes 0 .. steps + 1, as shares of the scale."""
    f = np.arange(steps + 2, dtype=f32) * f32(1 / steps)
    f = f * f
    return f if steps == 127 else f * f


def unbiased(x, steps, u):
    g = values(steps)
    c = np.searchsorted(g[1:steps + 1], x, side="right")
    return np.minimum(c + (x - g[c] > u * (g[c + 1] - g[c])), steps)


def nearest(x, steps):
    f = (np.arange(steps, dtype=f32) + f32(0.5)) * f32(1 / steps)
    f = f * f
    return np.searchsorted(f if steps == 127 else f * f, x, side="right")


def rounded(x, steps, u):
    """Signed codes and scales of the blocks of x; u None: nearest."""
    pad = -len(x) % 256
    b = np.concatenate([x, np.zeros(pad, f32)]).reshape(-1, 256)
    top = np.abs(b).max(1)
    scale = np.where(top < f32(2.0 ** -126), f32(0), top).astype(f32)
    with np.errstate(divide="ignore"):
        share = np.abs(b) * np.where(scale > 0, f32(1) / scale, f32(0))[:, None].astype(f32)
    if u is None:
        c = nearest(share, steps)
    else:
        c = unbiased(share, steps, np.concatenate([u, np.full(pad, 0.5, f32)]).reshape(-1, 256))
    if steps == 255:
        c = np.where((b > 0) & (scale > 0)[:, None], np.maximum(c, 1), 0)
    return np.where(b < 0, -c, c).ravel()[: len(x)], scale


def value_of(c, scale, steps):
    f = c.astype(f32) * f32(1 / steps)
    s = np.repeat(scale, 256)[: len(c)]
    return s * (f * np.abs(f)) if steps == 127 else s * ((f * f) * (f * f))


class Definition:
    """States of one tensor and their step."""

    def __init__(self, n, tensor=0, seed=1):
        self.m, self.v, self.tensor, self.seed = np.zeros(n, np.int64), np.zeros(n, np.int64), tensor, seed
        self.ms = self.vs = np.zeros(-(-n // 256), f32)

    def decoded(self):
        return value_of(self.m, self.ms, 127), value_of(self.v, self.vs, 255)

    def step(self, g, t, first=0):
        m, v = self.decoded()
        m = m * f32(B1) + g * f32(1 - B1)
        v = v * f32(B2) + (g * g) * f32(1 - B2)
        um = uv = None
        if self.seed:
            h = draws(self.seed, t, self.tensor, first + np.arange(len(g), dtype=u64))
            um, uv = unit(h), unit(reversed_bits(h))
        (self.m, self.ms), (self.v, self.vs) = rounded(m, 127, um), rounded(v, 255, uv)


# ---- on the host: the definition itself ----------------------------------------------------------------------------
@pytest.mark.parametrize("seed,step,tensor", [(1, 1, 0), (1, 2, 557), (2 ** 32 - 1, 2 ** 33 + 5, 3)])
def test_draws_are_uniform_and_independent(seed, step, tensor):
    n = 1 << 20
    i = np.arange(n, dtype=u64)
    h = draws(seed, step, tensor, i)
    m, v = unit(h).astype(np.float64), unit(reversed_bits(h)).astype(np.float64)
    later, other, far = (unit(x).astype(np.float64) for x in (draws(seed, step + 1, tensor, i), draws(seed, step, tensor + 1, i), draws(seed, step, tensor, i + u64(1 << 32))))
    for a, b in ((m, v), (m[1:], m[:-1]), (v[1:], v[:-1]), (m[256:], m[:-256]), (m, later), (m, other), (m, far)):
        cells = np.bincount((a * 64).astype(int) * 64 + (b * 64).astype(int), minlength=4096)
        chi2 = ((cells - len(a) / 4096) ** 2 / (len(a) / 4096)).sum()
        assert abs(chi2 - 4095) <= 6 * np.sqrt(2 * 4095), chi2                  # six deviations
        assert abs(np.corrcoef(a, b)[0, 1]) <= 6 / np.sqrt(len(a))
    assert 0 < m.min() < 1e-4 and 1 - 1e-4 < m.max() < 1


@pytest.mark.parametrize("steps", [127, 255])
def test_the_mean_is_the_value(steps):
    g = values(steps).astype(np.float64)
    rng = np.random.default_rng(steps)
    x = np.concatenate([rng.random(500) ** 4, [1.0, 0.5, g[2], g[steps - 1]]]).astype(f32)
    x = np.maximum(x, f32(g[1]))
    n = 4000
    c = np.stack([unbiased(x, steps, unit(draws(3, t, 0, np.arange(len(x))))) for t in range(1, n + 1)])
    lo = np.searchsorted(g[1:steps + 1], x, side="right")
    gap = g[lo + 1] - g[lo]
    assert ((c == lo) | (c == lo + 1)).all() and (c <= steps).all()
    assert (np.abs(g[c].mean(0) - x) <= 6 * gap / 2 / np.sqrt(n) + 1e-12).all()    # a two-valued draw deviates by half its gap at most
    assert (c[:, x == f32(g[2])] == 2).all()                                       # a value of the grid stays


def run(make_step, steps):
    """One block; gradients of normal size, those of the first 64 fall tenfold and of the next 64 become zero after 1000 steps."""
    rng = np.random.default_rng(7)
    base = np.exp(rng.uniform(-2, 0, 256))
    base[:128], base[255] = 0.5, 1
    m, v = np.zeros(256), np.zeros(256)
    for t in range(1, steps + 1):
        size = base.copy()
        if t > 1000:
            size[:64] *= 0.1
            size[64:128] = 0
        g = (rng.standard_normal(256) * size).astype(f32)
        m, v = B1 * m + (1 - B1) * g.astype(np.float64), B2 * v + (1 - B2) * g.astype(np.float64) ** 2
        make_step(g, t)
    return m, v


def check_long_run(m8, v8, v):
    """Codes of the fallen are at least 255 sqrt(sqrt(0.05^2 / 2)) = 48 (the block's largest v is below 2): spread 0.2 and less, of a median
    of 64 1.25 / 8 of that.  0.75 .. 1.33 is seven deviations and more."""
    for part in (slice(0, 64), slice(128, 255)):
        assert 0.75 <= np.median(v8[part] / v[part]) <= 1.33, (part, np.median(v8[part] / v[part]))
    assert not m8[64:128].any()


def test_unbiased_states_follow_the_gradients_over_a_long_run():
    d = Definition(256)
    _, v = run(d.step, 7000)
    check_long_run(*d.decoded(), v)


def test_nearest_states_freeze():
    """What the unbiased rounding is for: the definition of the nearest codes, on the same gradients."""
    d = Definition(256, seed=0)
    _, v = run(d.step, 7000)
    m8, v8 = d.decoded()
    assert np.median(v8[:64] / v[:64]) > 30 and np.median(v8[64:128] / v[64:128]) > 30 and m8[64:128].any()


def test_twelve_thousand_steps_of_stationary_and_of_rising_gradients():
    """A block of normal gradients of sizes e^-4 .. 1: codes from about 30 on, spread 0.26 and less, of a median of 256 1.25 / 16 of that and of
    the smallest 64 1.25 / 8.  And one of constant gradients, 64 of which rise from 0.2 to 0.6 beside a 1: code 197, spread 0.1, of a mean of 64
    an eighth; with nearest codes they stay at their old second moments, a ninth of the new."""
    rng = np.random.default_rng(11)
    size = np.exp(rng.uniform(-4, 0, 256))
    still, rising, frozen = Definition(256), Definition(256, 1), Definition(256, 1, seed=0)
    v, w = np.zeros(256), np.zeros(256)
    for t in range(1, 12_001):
        g = (rng.standard_normal(256) * size).astype(f32)
        v = B2 * v + (1 - B2) * g.astype(np.float64) ** 2
        still.step(g, t)
        r = np.full(256, 0.3, f32)
        r[:64], r[255] = 0.2 if t <= 1000 else 0.6, 1
        w = B2 * w + (1 - B2) * r.astype(np.float64) ** 2
        rising.step(r, t)
        frozen.step(r, t)
        if t in (1000, 4000, 12_000):
            q = still.decoded()[1] / v
            assert 0.9 <= np.median(q) <= 1.1 and 0.75 <= np.median(q[np.argsort(size)[:64]]) <= 1.33, (t, np.median(q))
    assert 0.9 <= (rising.decoded()[1] / w)[:64].mean() <= 1.1
    assert (frozen.decoded()[1] / w)[:64].mean() < 0.3


def test_seeds_have_32_bits():
    for seed in (-1, 1 << 32):
        with pytest.raises(ValueError, match="rounding_seed"):
            B.gnn_adamw_step(None, 1e-3, rounding_seed=seed)


# ---- on the GPU ------------------------------------------------------------------------------------------------------
def entry(n, pdt=torch.float32):
    z = lambda k, dtype: torch.zeros(k, dtype=dtype, device="cuda")
    blocks = -(-n // 256)
    return {"grad": z(n, torch.float32), "param": z(n, pdt), "m": z(n, torch.int8), "v": z(n, torch.uint8), "m_scale": z(blocks, torch.float32),
            "v_scale": z(blocks, torch.float32)}


def same(e, d):
    for key, want in (("m", d.m), ("v", d.v), ("m_scale", d.ms), ("v_scale", d.vs)):
        got = e[key].cpu().numpy()
        assert np.array_equal(got.astype(want.dtype), want), (key, np.flatnonzero(got != want)[:5])


@pytest.mark.gpu
@pytest.mark.parametrize("pdt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("seed", [1, 2 ** 32 - 1])
def test_codes_are_the_definitions(seed, pdt):
    """Every tensor of a table, over several steps, first with the number of the step from the host and then from the device."""
    sizes = [1, 255, 256, 257, 4097, 100_003]
    entries, defs = [entry(n, pdt) for n in sizes], [Definition(n, k, seed) for k, n in enumerate(sizes)]
    table, state = P.ParamTable(entries), P.StepState(6)
    rng = np.random.default_rng(seed)
    for t in range(1, 13):
        for e, d in zip(entries, defs):
            g = (rng.standard_normal(len(d.m)) * np.exp(rng.uniform(-8, 0, len(d.m)))).astype(f32)
            g[rng.random(len(g)) < 0.1] = 0
            e["grad"].copy_(torch.from_numpy(g))
            d.step(g, t)
        if t <= 6:
            P.gnn_adamw_step(table, 1e-3, (B1, B2), 1e-8, step=t, rounding_seed=seed)
        else:
            P.gnn_grad_norm(table, state)
            P.gnn_adamw_step(table, 1e-3, (B1, B2), 1e-8, state=state, rounding_seed=seed)
        for e, d in zip(entries, defs):
            same(e, d)


@pytest.mark.gpu
def test_elements_beyond_32_bits_draw_for_themselves():
    n, far = 2 ** 32 + 1000, 2 ** 32
    g = np.random.default_rng(1).standard_normal(1000).astype(f32)
    e = entry(n, torch.bfloat16)
    e["grad"][far:] = torch.from_numpy(g).cuda()
    d = Definition(1000, 0, 9)
    for t in (1, 2, 3):
        P.gnn_adamw_step(P.ParamTable([e]), 1e-3, (B1, B2), 1e-8, step=t, rounding_seed=9)
        d.step(g, t, first=far)
    same({"m": e["m"][far:], "v": e["v"][far:], "m_scale": e["m_scale"][far // 256:], "v_scale": e["v_scale"][far // 256:]}, d)
    assert not e["m"][:1 << 20].any() and not e["v"][:1 << 20].any()


@pytest.mark.gpu
def test_states_that_adamw_makes_follow_the_gradients_over_a_long_run():
    n = 4096      # the smallest tensor that gets 8-bit states; sixteen equal blocks, and the last of them looked at as well
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt = P.AdamW([{"param": p, "grad": g}], bits=8)

    def step(grads, t):
        g.copy_(torch.from_numpy(np.tile(grads, n // 256)))
        opt.step()
    _, v = run(step, 7000)
    e = opt.table.entries[0]
    assert e["m"].dtype == torch.int8 and opt.rounding_seed == 1
    m8, v8 = (x.cpu().numpy() for x in P.gnn_adamw_state_values(e["m"], e["m_scale"], e["v"], e["v_scale"]))
    for k in (0, 15):
        check_long_run(m8[256 * k:256 * k + 256], v8[256 * k:256 * k + 256], v)
    assert not np.array_equal(v8[:256], v8[-256:])      # blocks draw for themselves


@pytest.mark.gpu
def test_which_rounding_adamw_takes():
    """States made here: unbiased; given 8-bit states: nearest unless a seed is given; 32-bit states have no rounding."""
    new = lambda n: {"param": torch.zeros(n, device="cuda"), "grad": torch.zeros(n, device="cuda")}
    assert P.AdamW([new(4096)], bits=8).rounding_seed == 1 and P.AdamW([new(4096)], bits=8, rounding_seed=0).rounding_seed == 0
    assert P.AdamW([entry(300)]).rounding_seed == 0 and P.AdamW([entry(300), new(5000)], bits=8).rounding_seed == 0
    assert P.AdamW([entry(300)], rounding_seed=5).rounding_seed == 5
    assert P.AdamW([new(5000)]).rounding_seed == 0 and P.AdamW([new(100)], bits=8).rounding_seed == 0 and P.AdamW([]).rounding_seed == 0


@pytest.mark.gpu
def test_replays_of_a_captured_step_draw_anew():
    both = []
    for _ in range(2):
        p, g = torch.zeros(70_000, device="cuda"), torch.randn(70_000, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
        both.append((P.AdamW([{"param": p, "grad": g}], bits=8), p, g))
    (opt, p, g), (eager, q, k) = both
    for o in (opt, eager):
        o.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for _ in range(4):
        g.mul_(-0.7), k.mul_(-0.7)
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        for key in ("param", "m", "v", "m_scale", "v_scale"):
            assert torch.equal(opt.table.entries[0][key], eager.table.entries[0][key]), key
