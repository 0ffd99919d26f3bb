"""AdamW over many tensors against the formula in 64 bits, and, for what is held in 8 bits, against every operation rounded to fp32 in
numpy (a code is a choice between two neighbours that one rounding can turn).

Bounds, in roundings of u = 2^-24: m 4 (the gradient's scale, the factor's own, product, sum), v 6 (the scale twice, the square, the
factor's own, product, sum).  p: 3 of |p| (1 - lr wd itself, the product, the difference); the update m's own and 15 of itself (3 from v
under the root, the root, its factor and their product, eps and the sum, the quotient 4: it is within 2 ulp, the rate and its product,
the difference); in bf16 half a step, 2^-8 |p|, more."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZES = [1, 2, 3, 255, 256, 257, 0, 1000, 2047, 2048, 2049, 4096, 5, 12289, 100_003]
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.05)


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def tensors(sizes, p_type, g_type, eight, off=0, seed=0):
    """Parameters, gradients and states on the device, `off` values behind an allocation's start."""
    g = torch.Generator().manual_seed(seed)
    make = lambda t: (lambda r: r[off:off + t.numel()].copy_(t))(torch.zeros(t.numel() + off, dtype=t.dtype, device="cuda"))   # noqa: E731
    rnd = lambda n: torch.randn(n, generator=g)   # noqa: E731
    x = {"p": [make((rnd(n) * 0.1).to(p_type)) for n in sizes], "g": [make((rnd(n) * 10 ** (i % 7 - 5)).to(g_type)) for i, n in enumerate(sizes)]}
    x["copy"] = [make(torch.zeros(n, dtype=torch.bfloat16)) for n in sizes]
    if eight:
        scales = [-(-n // 256) for n in sizes]
        x["m"] = [make((rnd(n) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)) for n in sizes]
        x["r"] = [make((rnd(n).abs() * 100 + 0.01).clamp(0, 448).to(torch.float8_e4m3fn)) for n in sizes]
        x["ms"] = [torch.rand(n, generator=g).cuda() * 10.0 ** (i % 7 - 8) for i, n in enumerate(scales)]
        x["rs"] = [torch.rand(n, generator=g).cuda() * 10.0 ** (i % 7 - 7) for i, n in enumerate(scales)]
    else:
        x["m"] = [make(rnd(n) * 0.01) for n in sizes]
        x["v"] = [make(rnd(n).square() * 1e-4) for n in sizes]
    return x


def plan_of(pkg, x, copies=True):
    eight = "r" in x
    return pkg.new_adamw_plan(x["p"], x["g"], x["m"], x["r"] if eight else x["v"], x.get("ms"), x.get("rs"), x["copy"] if copies else None)


def held(codes, scales, n):
    return codes.float().cpu() * scales.cpu().repeat_interleave(256)[:n]


def formula(p, g, m, v, t, grad_scale, lr, beta1, beta2, eps, weight_decay):
    p, g, m, v = (a.double().cpu() for a in (p, g, m, v))
    g = g * grad_scale
    m2, v2 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    up = lr / (1 - beta1 ** t) * m2 / (v2.sqrt() / math.sqrt(1 - beta2 ** t) + eps)
    e_m = 4 * U * (beta1 * m.abs() + (1 - beta1) * g.abs()) + 1e-40
    e_v = 6 * U * v2 + 1e-40
    e_p = 3 * U * p.abs() + 15 * U * up.abs() + up.abs() * torch.where(m2 != 0, e_m / m2.abs().clamp(min=1e-300), 0.0) + 1e-40
    return p * (1 - lr * weight_decay) - up, m2, v2, e_p, e_m, e_v


def quantised(x, root):
    """e4m3 values and scale of one run of at most 256 fp32 values, in fp32 arithmetic."""
    top = np.float32(np.abs(x).max()) if x.size else np.float32(0)
    if not top >= np.float32(1e-30):
        return torch.zeros(x.size), 0.0
    y = x * (np.float32(448) * (np.float32(1) / top))
    if root:
        y = np.where((x > 0) & (y < np.float32(2 ** -9)), np.float32(2 ** -9), y)
    return torch.from_numpy(np.clip(y, -448, 448).astype(np.float32)).to(torch.float8_e4m3fn).float(), float(top * (np.float32(1) / np.float32(448)))


@pytest.mark.parametrize("off", [0, 1, 4])
@pytest.mark.parametrize("eight", [False, True], ids=["fp32", "e4m3"])
@pytest.mark.parametrize("g_type", DTYPES)
@pytest.mark.parametrize("p_type", DTYPES)
def test_step(pkg, p_type, g_type, eight, off):
    x = tensors(SIZES, DTYPES[p_type], DTYPES[g_type], eight, off, seed=off)
    old = {k: [t.clone() for t in ts] for k, ts in x.items()}
    plan = plan_of(pkg, x, copies=p_type == "fp32")
    pkg.esc_adamw_step(plan, 3, grad_scale=0.5, **HYPER)
    torch.cuda.synchronize()
    f = np.float32
    for i, n in enumerate(SIZES):
        m = held(old["m"][i], old["ms"][i], n) if eight else old["m"][i].cpu()
        v = held(old["r"][i], old["rs"][i], n).square() if eight else old["v"][i].cpu()
        p2, m2, v2, e_p, e_m, e_v = formula(old["p"][i], old["g"][i], m, v, 3, 0.5, **HYPER)
        far = e_p + (2.0 ** -8 * p2.abs() if p_type == "bf16" else 0)
        assert ((x["p"][i].double().cpu() - p2).abs() <= far).all(), (n, "p")
        if p_type == "fp32":
            assert torch.equal(x["copy"][i], x["p"][i].bfloat16())
        else:
            assert (x["copy"][i] == 0).all()
        if not eight:
            assert ((x["m"][i].double().cpu() - m2).abs() <= e_m).all() and ((x["v"][i].double().cpu() - v2).abs() <= e_v).all(), (n, "moments")
            continue
        gn = old["g"][i].float().cpu().numpy() * f(0.5)
        mn = m.numpy() * f(0.9) + gn * f(1 - 0.9)
        rn = np.sqrt(v.numpy() * f(0.99) + gn * gn * f(1 - 0.99))
        assert mn.dtype == rn.dtype == np.float32
        for name, scales, y in (("m", "ms", mn), ("r", "rs", rn)):
            for b in range(0, n, 256):
                codes, scale = quantised(y[b:b + 256], name == "r")
                assert float(x[scales][i][b // 256]) == scale, (n, name, b)
                assert torch.equal(x[name][i][b:b + 256].float().cpu(), codes), (n, name, b)
    # nothing beside the tensors was written
    for k in ("p", "g", "m"):
        for t in x[k]:
            if off and t.numel():
                base = torch.as_strided(t.view(torch.uint8), (off * t.element_size(),), (1,), 0)
                assert (base == 0).all()


@pytest.mark.parametrize("eight", [False, True], ids=["fp32", "e4m3"])
def test_many_steps_follow_the_formula(pkg, eight):
    """20 steps from zero states.  fp32 states against 64 bits.  8 bits: the first step's update is made before anything is rounded, so it
    is the formula's; later ones differ by what the states are off: m and r by 2^-4 of themselves a step at most."""
    sizes = [300, 5000]
    x = tensors(sizes, torch.float32, torch.float32, eight, seed=5)
    for k in ("m", "r", "v", "ms", "rs"):
        for t in x.get(k, []):
            t.zero_()
    plan = plan_of(pkg, x)
    p = [t.double().cpu() for t in x["p"]]
    m, v = [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]
    g = torch.Generator().manual_seed(9)
    for t in range(1, 21):
        for a in x["g"]:
            a.copy_(torch.randn(a.numel(), generator=g) * 1e-3 + 1e-3)
        pkg.esc_adamw_step(plan, t, **HYPER)
        for i in range(2):
            p[i], m[i], v[i], *_ = formula(p[i], x["g"][i], m[i], v[i], t, 1.0, **HYPER)
            err = (x["p"][i].double().cpu() - p[i]).abs()
            if not eight or t == 1:
                assert (err <= t * 40 * U * (p[i].abs() + HYPER["lr"] * 4)).all(), (t, float(err.max()))
            else:
                assert torch.isfinite(x["p"][i]).all() and (err <= t * HYPER["lr"] * 0.5).all(), (t, float(err.max()))


def test_scalars_and_skip_in_a_replayed_graph(pkg):
    x = tensors([700, 3000], torch.float32, torch.bfloat16, False, seed=2)
    start = {k: [t.clone() for t in ts] for k, ts in x.items()}
    plan = plan_of(pkg, x)
    scalars, skip = torch.zeros(4, device="cuda"), torch.zeros((), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        pkg.esc_adamw_step(plan, 1, scalars=scalars, skip=skip, **HYPER)
    for t, lr in ((1, 1e-2), (2, 3e-3)):
        scalars.copy_(torch.tensor(pkg.esc_adamw_scalars(t, lr, 0.9, 0.99, 0.05, 2.0)))
        graph.replay()
    skip.fill_(1)
    torch.cuda.synchronize()
    seen = [t.clone() for t in x["p"] + x["m"] + x["v"] + x["copy"]]
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(seen, x["p"] + x["m"] + x["v"] + x["copy"]))
    plan2 = plan_of(pkg, start)
    for t, lr in ((1, 1e-2), (2, 3e-3)):
        pkg.esc_adamw_step(plan2, t, **(HYPER | {"lr": lr}), grad_scale=2.0)
    for k in ("p", "m", "v", "copy"):
        assert all(torch.equal(a, b) for a, b in zip(x[k], start[k])), k


def test_a_captured_plan_is_refused(pkg):
    x = tensors([700], torch.float32, torch.float32, False)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        with pytest.raises(pkg.EscError):
            plan_of(pkg, x)
        torch.zeros(1, device="cuda")


@pytest.mark.parametrize("eight", [False, True], ids=["fp32", "e4m3"])
def test_non_finite_gradients_stay_where_they_are(pkg, eight):
    x = tensors([1024], torch.float32, torch.float32, eight, seed=3)
    y = {k: [t.clone() for t in ts] for k, ts in x.items()}
    x["g"][0][300], x["g"][0][700] = math.nan, math.inf
    pkg.esc_adamw_step(plan_of(pkg, x), 5, **HYPER)
    pkg.esc_adamw_step(plan_of(pkg, y), 5, **HYPER)
    hit = torch.zeros(1024, dtype=torch.bool, device="cuda")
    hit[300] = hit[700] = True
    assert torch.isnan(x["p"][0][hit]).all() and torch.equal(x["p"][0][~hit], y["p"][0][~hit])
    assert torch.isnan(x["m"][0].float()[300])
    scales = torch.cat([x[k][0] for k in ("ms", "rs")]) if eight else torch.zeros(1)
    assert torch.isfinite(scales).all()


def test_zero_and_tiny_states_in_eight_bits(pkg):
    """A run of zeros has scale zero; a root far below its neighbours is kept at the smallest value, not at zero."""
    x = tensors([512], torch.float32, torch.float32, True, seed=4)
    for k in ("m", "r", "ms", "rs"):
        x[k][0].zero_()
    g = x["g"][0]
    g.zero_()
    g[256:] = 1e-9
    g[256] = 1.0
    pkg.esc_adamw_step(plan_of(pkg, x), 1, **HYPER)
    r = x["r"][0].float()
    assert float(x["rs"][0][0]) == 0 and float(x["ms"][0][0]) == 0 and (r[:256] == 0).all()
    assert float(r[256]) == 448 and (r[257:] == 2.0 ** -9).all() and (x["m"][0].float()[257:] == 0).all()
    assert torch.isfinite(x["p"][0]).all()
    g.zero_()
    before = x["p"][0].clone()
    pkg.esc_adamw_step(plan_of(pkg, x), 2, **HYPER)
    moved = (x["p"][0] - before * (1 - HYPER["lr"] * HYPER["weight_decay"])).abs()
    assert (moved <= 2 * HYPER["lr"]).all(), float(moved.max())


def test_refuses(pkg):
    x = tensors([64, 65], torch.float32, torch.float32, False)
    with pytest.raises(ValueError):
        pkg.new_adamw_plan(x["p"], x["g"][:1], x["m"], x["v"])
    with pytest.raises(ValueError):
        pkg.new_adamw_plan(x["p"], [t.bfloat16() if i else t for i, t in enumerate(x["g"])], x["m"], x["v"])
    with pytest.raises(ValueError):
        pkg.new_adamw_plan(x["p"], x["g"], x["m"], x["v"], [torch.zeros(1, device="cuda")] * 2, [torch.zeros(1, device="cuda")] * 2)
    with pytest.raises(TypeError):
        pkg.new_adamw_plan(x["p"], x["g"], [t.bfloat16() for t in x["m"]], x["v"])
    with pytest.raises(ValueError):
        pkg.new_adamw_plan(x["p"], x["g"], x["m"], [t.cpu() for t in x["v"]])
    with pytest.raises(pkg.EscError):
        pkg.esc_adamw_step(plan_of(pkg, x), 0, lr=1e-3)
