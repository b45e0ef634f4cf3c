"""GPU: gradient norm and AdamW over many tensors against the formulas in 64 bits, 8-bit states against their definition bit by bit.

Tolerances count roundings of u = 2^-24 (float), half a step each, as derived at each check.  The definition of the 8-bit codes fixes
every 32-bit operation, so codes and scales have to be equal to numpy's, not near."""
import math

import numpy as np
import pytest
import torch

import paper_2311_06837_amd as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
f32 = np.float32


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def m_values(c, scale):
    f = c.astype(f32) * f32(1 / 127)
    return scale * (f * np.abs(f))


def v_values(c, scale):
    f = c.astype(f32) * f32(1 / 255)
    f = f * f
    return scale * (f * f)


def blocks_of(x):
    pad = -len(x) % 256
    return np.concatenate([x, np.zeros(pad, x.dtype)]).reshape(-1, 256)


def codes_of(x, steps):
    """Codes and scales by the definition, in float32."""
    b = blocks_of(x.astype(f32))
    top = np.abs(b).max(1)
    bad = ~np.isfinite(b).all(1)
    scale = np.where(top < f32(2.0 ** -126), f32(0), top).astype(f32)
    with np.errstate(divide="ignore", invalid="ignore"):
        share = np.abs(b) * np.where(scale > 0, f32(1) / scale, f32(0))[:, None].astype(f32)
    f = (np.arange(steps, dtype=f32) + f32(0.5)) * f32(1 / steps)
    borders = f * f
    if steps == 255:
        borders = borders * borders
    c = np.searchsorted(borders, np.where(np.isnan(share), f32(0), share).ravel(), side="right").reshape(b.shape)
    if steps == 255:
        c = np.where((b > 0) & (scale > 0)[:, None], np.maximum(c, 1), c)
    else:
        c = np.where(b < 0, -c, c)
    c[bad] = 0
    scale[bad] = np.nan
    return c.ravel()[: len(x)], scale


def one(rng, n, pdt="f32", gdt="f32", bits=32, decay=0.01, shift=0, size=1e-2):
    """A tensor with a past: host values and the device entry.  shift: elements by which every array is off its allocation."""
    def dev(a, dtype):
        t = torch.zeros(n + shift, dtype=dtype, device="cuda")
        t[shift:] = torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()
        return t[shift:]
    h = {"p": rng.standard_normal(n).astype(f32) * f32(0.1), "g": rng.standard_normal(n).astype(f32) * f32(size), "bits": bits, "decay": decay, "pdt": pdt}
    h["g"] = bf16(h["g"]) if gdt == "bf16" else h["g"]
    h["p"] = bf16(h["p"]) if pdt == "bf16" else h["p"]
    m = (rng.standard_normal(n) * 0.3 * size).astype(f32)
    v = ((rng.standard_normal(n) * size) ** 2).astype(f32)
    T = {"f32": torch.float32, "bf16": torch.bfloat16}
    e = {"grad": dev(h["g"], T[gdt]), "param": dev(h["p"], torch.bfloat16 if pdt != "f32" else torch.float32), "weight_decay": decay}
    if pdt == "master":
        e["master"] = dev(h["p"], torch.float32)
    if bits == 32:
        h["m"], h["v"] = m, v
        e["m"], e["v"] = dev(m, torch.float32), dev(v, torch.float32)
    else:
        (mc, ms), (vc, vs) = codes_of(m, 127), codes_of(v, 255)
        h["m"], h["v"] = blocks_of(mc.astype(f32)), blocks_of(vc.astype(f32))
        h["m"], h["v"] = m_values(h["m"], ms[:, None]).ravel()[:n], v_values(h["v"], vs[:, None]).ravel()[:n]
        e["m"], e["v"] = dev(mc, torch.int8), dev(vc, torch.uint8)
        e["m_scale"], e["v_scale"] = torch.from_numpy(ms).cuda(), torch.from_numpy(vs).cuda()
    return h, e


HYP = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8)


def check_update(h, e, coef, step, hyp=HYP):
    """One step by the formula in 64 bits (moments also in 32, operation by operation); compares what the device wrote."""
    (b1, b2), lr, eps = hyp["betas"], hyp["lr"], hyp["eps"]
    c32 = f32(coef)
    g = h["g"] * c32
    m = h["m"] * f32(b1) + g * f32(1 - b1)
    v = h["v"] * f32(b2) + (g * g) * f32(1 - b2)
    assert m.dtype == v.dtype == np.float32
    # in 64 bits
    G = h["g"].astype(np.float64) * coef
    M = h["m"].astype(np.float64) * b1 + G * (1 - b1)
    V = h["v"].astype(np.float64) * b2 + G * G * (1 - b2)
    den = np.sqrt(V / (1 - b2 ** step)) + eps
    upd = lr / (1 - b1 ** step) * M / den
    want = h["p"].astype(np.float64) * (1 - lr * h["decay"]) - upd
    host = lambda t: t.float().cpu().numpy()
    if h["bits"] == 32:
        assert np.array_equal(host(e["m"]), m) and np.array_equal(host(e["v"]), v)
    else:
        for key, x, steps in (("m", m, 127), ("v", v, 255)):
            c, s = codes_of(x, steps)
            assert np.array_equal(e[key + "_scale"].cpu().numpy(), s, equal_nan=True), key + "_scale"
            assert np.array_equal(e[key].cpu().numpy().astype(np.int64), c), key
    # moments against 64 bits: m two products and coefficients (3 u each of its two terms) and a sum; v 6 u of its sum of non-negative terms
    m_err = U * (4 * np.abs(h["m"] * b1) + 5 * np.abs(G * (1 - b1)))
    assert (np.abs(m - M) <= m_err + 1e-45).all() and (np.abs(v - V) <= 8 * U * V + 1e-45).all()
    # parameter: the decayed weight (factor and product, u each), the update (error of m; v by half; root, quotient, product, sum: at most
    # 12 u with roots and quotients good to 2 u), the last sum u
    p_err = U * (2 * np.abs(h["p"]) + 12 * np.abs(upd) + np.abs(want) + np.abs(upd)) + lr / (1 - b1 ** step) * m_err / den
    got = host(e["master"] if "master" in e else e["param"])
    if h["pdt"] == "bf16":
        p_err = p_err + 2.0 ** -8 * np.abs(want) * (1 + U)
    bad = np.abs(got - want) > p_err + 1e-45
    assert not bad.any(), (np.flatnonzero(bad)[:5], got[bad][:5], want[bad][:5])
    if "master" in e:
        assert torch.equal(e["param"], e["master"].to(torch.bfloat16))


def run(pairs, max_norm=0.0, step=7, grad_scale=1.0):
    table, state = P.ParamTable([e for _, e in pairs]), P.StepState(step - 1)
    P.gnn_grad_norm(table, state, grad_scale, max_norm)
    P.gnn_adamw_step(table, HYP["lr"], HYP["betas"], HYP["eps"], state=state)
    norm = abs(grad_scale) * math.sqrt(sum(float(np.sum(h["g"].astype(np.float64) ** 2)) for h, _ in pairs))
    assert abs(state.norm.item() - norm) <= 2 * U * norm      # one rounding; the sum in 64 bits is far below
    coef = grad_scale * (max_norm / norm if max_norm > 0 and norm > max_norm else 1.0)
    assert abs(state.coef.item() - coef) <= 2 * U * abs(coef)
    assert state.step.item() == step and state.ok.item() == 1 and state.skipped.item() == 0
    for h, e in pairs:
        check_update(h, e, coef if max_norm == 0 or norm <= max_norm else state.coef.item(), step)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdt", ["f32", "bf16", "master"])
@pytest.mark.parametrize("gdt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 255, 4097])
def test_one_tensor(bits, pdt, gdt, n):
    print(f"adamw: n={n} {pdt} {gdt} {bits} bits", flush=True)
    run([one(np.random.default_rng(n), n, pdt, gdt, bits)])


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("max_norm", [0.0, 0.05, 1e9])
def test_tensors_of_all_kinds_in_one_table(shift, max_norm):
    rng = np.random.default_rng(3)
    sizes = [1, 2, 3, 0, 255, 256, 257, 4095, 4096, 4097, 0, 10001, 20000, 41, 0]
    pairs = [one(rng, n, rng.choice(["f32", "bf16", "master"]), rng.choice(["f32", "bf16"]), int(rng.choice([8, 32])), float(rng.choice([0, 0.1])), shift)
             for n in sizes * 2]
    run(pairs, max_norm, step=1, grad_scale=0.5)


def test_more_tensors_than_a_search_level():
    rng = np.random.default_rng(5)
    run([one(rng, int(rng.integers(1, 700)), bits=int(rng.choice([8, 32]))) for _ in range(4200)], 1.0)


def test_more_chunks_than_workgroups():
    rng = np.random.default_rng(6)
    run([one(rng, 9_000_001, bits=8), one(rng, 300), one(rng, 700_000, "master")], 1.0)


@pytest.mark.parametrize("step", [1, 100, 10 ** 6])
def test_second_moments_below_the_normal_floats_divide(step):
    """Their root counts where eps is small: at eps = 1e-16 and the first steps 1 % of what divides.  The gradients are zero, so the new
    second moment is one product, in subnormals half a step of 2^-149 off; weights are zero, so that the update is what is compared."""
    rng = np.random.default_rng(21)
    n = 1000
    h, e = one(rng, n)
    h["p"][:], h["g"][:] = 0, 0
    h["v"] = (2.0 ** -rng.uniform(126.5, 140, n)).astype(f32)
    h["v"][::7] = f32(1e-6)       # ordinary ones and zeros beside them
    h["v"][::11] = 0
    h["m"] = (rng.standard_normal(n) * 1e-17).astype(f32)
    for key, name in (("p", "param"), ("g", "grad"), ("m", "m"), ("v", "v")):
        e[name].copy_(torch.from_numpy(h[key]))
    eps = float(f32(1e-16))
    P.gnn_adamw_step(P.ParamTable([e]), 1e-3, HYP["betas"], eps, step=step)
    v = h["v"] * f32(0.999)       # what the state holds
    assert np.array_equal(e["v"].cpu().numpy(), v) and (v < 2.0 ** -126).sum() > n // 2
    upd = 1e-3 / (1 - 0.9 ** step) * 0.9 * h["m"].astype(np.float64) / (np.sqrt(v.astype(np.float64) / (1 - 0.999 ** step)) + eps)
    got = -e["param"].double().cpu().numpy()
    # coefficient of m, m, factor of the step, root and its factor (2 u for an ulp), their product, the sum, reciprocal, two products: 12 u
    assert (np.abs(got - upd) <= 12 * U * np.abs(upd)).all(), np.max(np.abs(got - upd) / np.maximum(np.abs(upd), 1e-60)) / U


@pytest.mark.parametrize("step", [1, 2, 1000, 10 ** 7])
def test_step_numbers(step):
    run([one(np.random.default_rng(1), 1000)], step=step)


def test_without_a_state_the_hosts_step_counts():
    h, e = one(np.random.default_rng(2), 5000, bits=8)
    P.gnn_adamw_step(P.ParamTable([e]), HYP["lr"], HYP["betas"], HYP["eps"], step=3, grad_scale=0.25)
    check_update(h, e, 0.25, 3)
    h, e = one(np.random.default_rng(2), 5000)
    lr = torch.tensor([HYP["lr"]], device="cuda")
    P.gnn_adamw_step(P.ParamTable([e]), 5.0, HYP["betas"], HYP["eps"], step=3, lr_device=lr)
    check_update(h, e, 1.0, 3, {**HYP, "lr": float(lr.item())})


@pytest.mark.parametrize("poison", [math.inf, -math.inf, math.nan])
def test_a_step_with_an_infinite_gradient_changes_nothing(poison):
    rng = np.random.default_rng(4)
    pairs = [one(rng, 300), one(rng, 5000, "master", bits=8)]
    pairs[1][1]["grad"][4999] = poison
    before = [{k: t.clone() for k, t in e.items() if torch.is_tensor(t)} for _, e in pairs]
    opt = P.AdamW([e for _, e in pairs], max_norm=1.0, step=4)
    opt.step()
    assert (opt.state.ok.item(), opt.state.step.item(), opt.state.skipped.item()) == (0, 4, 1)
    for (_, e), b in zip(pairs, before):
        for k, t in b.items():
            assert torch.equal(torch.nan_to_num(e[k].float(), 7.0), torch.nan_to_num(t.float(), 7.0)), k
    pairs[1][1]["grad"][4999] = 0.0
    opt.step()
    assert (opt.state.ok.item(), opt.state.step.item(), opt.state.skipped.item()) == (1, 5, 1)


@pytest.mark.parametrize("grad_scale,refused", [(1.0, True), (-1.0, True), (0.25, False), (1e-3, False)])
def test_a_norm_that_is_no_float_refuses_the_step(grad_scale, refused):
    """Four gradients of 3e38 are finite, their norm of 6e38 is not a float: what is stored as infinite is not taken."""
    h, e = one(np.random.default_rng(22), 4)
    h["g"][:] = 3e38
    e["grad"].fill_(3e38)
    before = {k: e[k].clone() for k in ("param", "m", "v")}
    table, state = P.ParamTable([e]), P.StepState(6)
    P.gnn_grad_norm(table, state, grad_scale, 1.0)
    P.gnn_adamw_step(table, HYP["lr"], HYP["betas"], HYP["eps"], state=state)
    assert math.isinf(state.norm.item()) == refused and state.ok.item() == (0 if refused else 1)
    assert (state.step.item(), state.skipped.item()) == ((6, 1) if refused else (7, 0))
    for k, t in before.items():
        assert torch.equal(e[k], t) == refused, k
    if not refused:
        check_update(h, e, state.coef.item(), 7)


def test_8_bit_blocks_of_zeros_tiny_values_and_nan():
    h, e = one(np.random.default_rng(8), 1024 + 7, bits=8)
    for key in ("m", "v"):
        e[key][:256], e[key + "_scale"][:1] = 0, 0.0
        h[key][:256] = 0
    for a, b in ((0, 256), (256, 512)):
        h["g"][a:b] = 0
        e["grad"][a:b] = 0
    h["g"][600], h["g"][1030] = np.nan, 1e-22        # the square of the second is below the smallest float
    e["grad"][600], e["grad"][1030] = math.nan, 1e-22
    P.gnn_adamw_step(P.ParamTable([e]), HYP["lr"], HYP["betas"], HYP["eps"], step=2)
    ms, vs = e["m_scale"].cpu(), e["v_scale"].cpu()
    assert ms[0] == 0 and vs[0] == 0 and not e["m"][:256].any() and not e["v"][:256].any()
    assert torch.isnan(ms[2]) and torch.isnan(vs[2]) and not e["m"][512:768].any()
    fine = [0, 1, 3, 4]
    assert torch.isfinite(ms[fine]).all() and torch.isfinite(vs[fine]).all()
    mv, vv = P.gnn_adamw_state_values(e["m"], e["m_scale"], e["v"], e["v_scale"])
    assert torch.isnan(mv[512:768]).all() and torch.isnan(mv).sum() == 256 and torch.isnan(vv).sum() == 256
    assert torch.isnan(e["param"]).sum() == 1       # the weight whose gradient was NaN


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 256, 4099])
def test_state_values(dtype, n):
    rng = np.random.default_rng(n)
    c, d = rng.integers(-127, 128, n).astype(np.int8), rng.integers(0, 256, n).astype(np.uint8)
    s, t = (rng.random(-(-n // 256)).astype(f32) for _ in range(2))
    m, v = P.gnn_adamw_state_values(*(torch.from_numpy(x).cuda() for x in (c, s, d, t)), dtype=dtype)
    want = m_values(blocks_of(c.astype(f32)), s[:, None]).ravel()[:n], v_values(blocks_of(d.astype(f32)), t[:, None]).ravel()[:n]
    for got, w in zip((m, v), want):
        assert torch.equal(got.cpu(), torch.from_numpy(w).to(dtype))


def test_8_bit_states_are_the_nearest_of_their_grid():
    """Against the formula in 64 bits: no value is further than half a step from what it stands for (a root's u is far below the steps)."""
    h, e = one(np.random.default_rng(9), 100_000, bits=8)
    P.gnn_adamw_step(P.ParamTable([e]), HYP["lr"], HYP["betas"], HYP["eps"], step=5)
    g = h["g"].astype(np.float64)
    for key, x, steps, power in (("m", 0.9 * h["m"] + 0.1 * g, 127, 2), ("v", 0.999 * h["v"] + 0.001 * g * g, 255, 4)):
        top = np.repeat(np.abs(blocks_of(x)).max(1), 256)[: len(x)]
        root = (np.abs(x) / top) ** (1 / power) * steps
        c = np.abs(e[key].cpu().numpy().astype(np.float64))
        assert (np.abs(c - root) <= 0.5 + 1e-4).all() or ((c == 1) & (root < 0.5))[np.abs(c - root) > 0.5 + 1e-4].all()
        assert (np.sign(e[key].cpu().numpy().astype(np.float64)) == np.sign(x) * (c > 0)).all()


def test_a_captured_step_follows_the_schedule_and_the_gradients():
    pairs = [one(np.random.default_rng(11), n, bits=b) for n, b in ((5000, 8), (300, 32), (70_000, 32))]
    twin = [{k: (t.clone() if torch.is_tensor(t) else t) for k, t in e.items()} for _, e in pairs]
    lr, lr2 = torch.tensor([1e-3], device="cuda"), torch.tensor([1e-3], device="cuda")
    opt, eager = P.AdamW([e for _, e in pairs], lr=lr, max_norm=0.1), P.AdamW(twin, lr=lr2, max_norm=0.1)
    for o in (opt, eager):
        o.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for k in range(4):
        for l in (lr, lr2):
            l.fill_(1e-3 / (k + 2))
        for (_, e), t in zip(pairs, twin):
            e["grad"].mul_(-0.7)
            t["grad"].mul_(-0.7)
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert opt.state.step.item() == eager.state.step.item() == k + 2
        for (_, e), t in zip(pairs, twin):
            for key in ("param", "m", "v"):
                assert torch.equal(e[key], t[key]), (k, key)


def test_on_another_stream():
    h, e = one(np.random.default_rng(12), 100_000, bits=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        opt = P.AdamW([e], **HYP)
        s.wait_stream(torch.cuda.default_stream())
        opt.step()
    s.synchronize()
    check_update(h, e, 1.0, 1)


def test_norm_alone_repeats_bit_for_bit():
    g = [torch.randn(n, device="cuda") for n in (1, 1000, 10_000_019)] + [torch.randn(77, device="cuda").bfloat16()]
    table, state = P.ParamTable([{"grad": t} for t in g]), P.StepState()
    got = []
    for _ in range(3):
        P.gnn_grad_norm(table, state, grad_scale=-2.0, max_norm=3.0)
        got.append((state.sum_sq.item(), state.norm.item(), state.coef.item()))
    assert got[0] == got[1] == got[2] and state.step.item() == 3
    want = 2 * math.sqrt(sum(t.double().square().sum().item() for t in g))
    assert abs(got[0][1] - want) <= 2 * U * want and got[0][2] < 0


def test_no_tensors():
    opt = P.AdamW([])
    opt.step()
    assert opt.state.step.item() == 1 and opt.state.norm.item() == 0.0


@pytest.mark.parametrize("bits", [8, 32])
def test_elements_beyond_32_bits(bits):
    """The last elements of a tensor of 2^31 + 1000 are updated as those of a small one, and nothing before them is touched."""
    n, far = 2 ** 31 + 1000, 2 ** 31
    h, e = one(np.random.default_rng(13), 1000, bits=bits)
    big = {"weight_decay": e["weight_decay"]}
    for key in ("param", "grad", "m", "v"):
        big[key] = torch.zeros(n, dtype=e[key].dtype, device="cuda")
        big[key][far:] = e[key]
    if bits == 8:
        for key in ("m_scale", "v_scale"):
            big[key] = torch.zeros((n + 255) // 256, device="cuda")
            big[key][far // 256:] = e[key]
    outs = []
    for t in (e, big):
        opt = P.AdamW([t], max_norm=1.0, **HYP)
        opt.step()
        outs.append((opt.state.norm.item(), opt.state.coef.item()))
    assert outs[0] == outs[1]
    for key in ("param", "m", "v"):
        assert torch.equal(big[key][far:], e[key]), key
        assert not big[key][:1 << 20].any() and not big[key][far - (1 << 20):far].any(), key
