"""The layers of an ESC block around its attention and convolutions, as cases that can be timed and compared.

An ESC block norms every pixel over its channels (layer norm) and maps pixels to pixels (the attention's one projection to q, k and
v, its output projection with the block's residual, the two 1x1 convolutions of the feed-forward network with a GELU between
them).  The operators here are that norm and that linear layer, each forward and backward.

  norm         y = (x - mean) / sqrt(var + eps) * weight + bias over the channels of every row
  norm_grad    the gradients of x (with the gradient that came round the layer added, where there is one), weight and bias
  linear       z = x weight^T + bias;  out = act(z) + residual;  z as it is too, where a backward pass will want it
  linear_grad  g = grad_out act'(z);  grad_x = g weight, grad_weight = g^T x, grad_bias = sum of g

Keys of a case: op; dtype ("fp32", "bf16") of all tensors; rows (pixels of all images), C channels of a norm or K inputs and N outputs
of a linear layer; "pad": values between the rows of x beyond its channels (x is then a slice of a wider tensor); "skip" (norm_grad)
or "residual" (linear): whether there is one; "act" ("none", "relu", "gelu"); "keep": whether linear writes z; "grads": type of the
weights' gradients.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def _norm(name, dtype, rows, C, pad=0):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "C": C, "pad": pad}


def _norm_grad(name, dtype, rows, C, skip, grads, pad=0):
    return {"name": name, "op": "norm_grad", "dtype": dtype, "rows": rows, "C": C, "skip": skip, "grads": grads, "pad": pad}


def _linear(name, dtype, rows, K, N, act="none", residual=False, keep=False, pad=0):
    return {"name": name, "op": "linear", "dtype": dtype, "rows": rows, "K": K, "N": N, "act": act, "residual": residual, "keep": keep, "pad": pad}


def _linear_grad(name, dtype, rows, K, N, act, grads, pad=0):
    return {"name": name, "op": "linear_grad", "dtype": dtype, "rows": rows, "K": K, "N": N, "act": act, "grads": grads, "pad": pad}


def listed():
    return [
        # one small crop at the small width (3 heads of 16): latency of a single call
        _norm("norm_fp32_crop_64x64x48", "fp32", 64 * 64, 48),
        # the LR map of x2 super-resolution to 1280x720
        _norm("norm_bf16_640x360x64", "bf16", 640 * 360, 64),
        # training: 64 patches of 64x64, with the residual's gradient added on the way
        _norm_grad("norm_grad_bf16_64x64x64x64", "bf16", 64 * 64 * 64, 64, True, "bf16"),
        # the large model on the LR map of x4, fine-tuned in fp32
        _norm_grad("norm_grad_fp32_320x180x192", "fp32", 320 * 180, 192, False, "fp32"),
        # q, k and v of every pixel by one projection
        _linear("qkv_bf16_640x360_64_192", "bf16", 640 * 360, 64, 192),
        # the large model's feed-forward network, first half, as a training step runs it: z is kept
        _linear("ffn_bf16_320x180_192_384", "bf16", 320 * 180, 192, 384, "gelu", keep=True),
        # x3, an odd width, in the precision the paper times: the attention's output projection with the residual
        _linear("proj_fp32_427x240_64_64", "fp32", 427 * 240, 64, 64, residual=True),
        # a few rows of a generic wide layer: latency, and the weights' bytes
        _linear("few_bf16_16_1024_4096", "bf16", 16, 1024, 4096, "gelu"),
        # sizes that no tile and no 16-byte piece divides, rows that are a slice of a wider tensor
        _linear("odd_bf16_10007_250_777", "bf16", 10007, 250, 777, "relu", residual=True, pad=3),
        # training: 64 patches of 64x64, first half of the feed-forward network
        _linear_grad("grad_bf16_64x64x64_64_128", "bf16", 64 * 64 * 64, 64, 128, "gelu", "bf16"),
        # the q, k and v projection at the small width, fine-tuned in fp32
        _linear_grad("grad_fp32_4x64x64_48_144", "fp32", 4 * 64 * 64, 48, 144, "none", "fp32"),
        # a generic wide layer: bound by its products
        _linear_grad("grad_bf16_16384_1024_4096", "bf16", 16384, 1024, 4096, "gelu", "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly whole heads of 16 channels, as networks have them; a third is any number."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.34 else max(16, (n + 8) // 16 * 16)


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "linear", "linear", "linear_grad", "linear_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    grads = "fp32" if dtype == "fp32" else "bf16"
    pad = rng.choice([0, 0, 0, 8, rng.randint(1, 40)])
    rows = _log_int(rng, 1, 260_000)
    if op in ("norm", "norm_grad"):
        C = _width(rng, 5, 4096)
        rows = max(1, min(rows, 40_000_000 // C))
        c = _norm("", dtype, rows, C, pad) if op == "norm" else _norm_grad("", dtype, rows, C, rng.random() < 0.5, grads, pad)
    else:
        K, N = _width(rng, 8, 4096), _width(rng, 8, 4096)
        most = (6e10 if op == "linear" else 3e10) * (0.2 if dtype == "fp32" else 1.0)    # products of two values
        rows = max(1, min(rows, int(most / (K * N)), 64_000_000 // max(K, N)))
        act = rng.choice(["none", "relu", "gelu"])
        if op == "linear":
            c = _linear("", dtype, rows, K, N, act, rng.random() < 0.5, act != "none" and rng.random() < 0.5, pad)
        else:
            c = _linear_grad("", dtype, rows, K, N, act, grads, pad)
    del c["name"]
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _features(case, width, g, dtype):
    """Rows as a residual stream has them: channels of different means and spreads, rows of different sizes; a slice where there is a pad."""
    rows, pad = case["rows"], case["pad"]
    x = torch.randn(rows, width + pad, generator=g, device="cuda")
    x *= torch.exp(torch.randn(width + pad, generator=g, device="cuda") * 0.3)
    x += torch.randn(width + pad, generator=g, device="cuda") * 0.5
    x *= torch.exp(torch.randn(rows, 1, generator=g, device="cuda") * 0.3)
    return x.to(dtype)[:, :width]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *n: torch.randn(*n, generator=g, device="cuda")       # noqa: E731
    new = lambda *n, t=None: torch.empty(*n, dtype=t or dtype, device="cuda")   # noqa: E731
    dtype, rows, op = DTYPES[case["dtype"]], case["rows"], case["op"]
    s = {"case": case, "scratch": {}}
    if op in ("norm", "norm_grad"):
        C = case["C"]
        s["x"] = _features(case, C, g, dtype)
        s["weight"], s["bias"] = (1 + 0.2 * rand(C)).to(dtype), (0.1 * rand(C)).to(dtype)
        if op == "norm":
            s["y"] = new(rows, C)
            return s
        s["gy"] = rand(rows, C).to(dtype)
        s["skip"] = rand(rows, C).to(dtype) if case["skip"] else None
        s["g_x"] = new(rows, C)
        s["g_weight"], s["g_bias"] = new(C, t=DTYPES[case["grads"]]), new(C, t=DTYPES[case["grads"]])
        return s
    K, N = case["K"], case["N"]
    s["x"] = _features(case, K, g, dtype)
    s["weight"], s["bias"] = (rand(N, K) * K ** -0.5).to(dtype), (0.1 * rand(N)).to(dtype)
    if op == "linear":
        s["residual"] = rand(rows, N).to(dtype) if case["residual"] else None
        s["out"], s["z"] = new(rows, N), new(rows, N) if case["keep"] else None
        return s
    s["go"] = rand(rows, N).to(dtype)
    s["z"] = (1.2 * rand(rows, N)).to(dtype) if case["act"] != "none" else None     # as the forward pass left it
    s["g_x"] = new(rows, K)
    s["g_weight"], s["g_bias"] = new(N, K, t=DTYPES[case["grads"]]), new(N, t=DTYPES[case["grads"]])
    return s


# ---- the operators' plain forms ---------------------------------------------------------------------------------------------


def _plain_norm(s):
    x = s["x"].float()
    x = x - x.mean(1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    return (x * s["weight"].float() + s["bias"].float()).to(s["x"].dtype)


def _plain_norm_grad(s):
    x, gy = s["x"].float(), s["gy"].float()
    x = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    x = x * r
    a = gy * s["weight"].float()
    g_x = (a - a.mean(1, keepdim=True) - x * (a * x).mean(1, keepdim=True)) * r
    if s["skip"] is not None:
        g_x = g_x + s["skip"].float()
    return {"g_x": g_x.to(s["x"].dtype), "g_weight": (gy * x).sum(0).to(s["g_weight"].dtype), "g_bias": gy.sum(0).to(s["g_bias"].dtype)}


def _plain_act(act, z):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    return 0.5 * z * torch.special.erfc(z * -math.sqrt(0.5)) if act == "gelu" else z


def _plain_act_grad(act, z):
    if act == "relu":
        return (z > 0).float()
    return 0.5 * torch.special.erfc(z * -math.sqrt(0.5)) + z * torch.exp(z * z * -0.5) * (1 / math.sqrt(2 * math.pi))


def _plain_linear(s):
    dtype = s["x"].dtype
    z = s["x"].float() @ s["weight"].float().t() + s["bias"].float()
    out = _plain_act(s["case"]["act"], z)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(dtype), "z": z.to(dtype)} if s["z"] is not None else {"out": out.to(dtype)}


def _plain_linear_grad(s):
    g = s["go"].float()
    if s["z"] is not None:
        g = g * _plain_act_grad(s["case"]["act"], s["z"].float())
    return {"g_x": (g @ s["weight"].float()).to(s["x"].dtype), "g_weight": (g.t() @ s["x"].float()).to(s["g_weight"].dtype),
            "g_bias": g.sum(0).to(s["g_bias"].dtype)}


# ---- one pass ---------------------------------------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(state, op)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "linear": _plain_linear, "linear_grad": _plain_linear_grad}[op](state)


def _run_own(s, op):
    import paper_2503_06671_b200 as esc

    case = s["case"]
    if op == "norm":
        return esc.esc_layer_norm_forward(s["x"], s["weight"], s["bias"], EPS, s["y"])
    if op == "norm_grad":
        if not s["scratch"]:
            s["scratch"]["ws"] = esc.new_layer_norm_workspace(case["rows"], case["C"])
        esc.esc_layer_norm_backward(s["x"], s["weight"], EPS, s["gy"], s["g_x"], s["g_weight"], s["g_bias"], s["skip"], s["scratch"]["ws"])
        return {k: s[k] for k in ("g_x", "g_weight", "g_bias")}
    act = {"none": esc.ESC_ACT_NONE, "relu": esc.ESC_ACT_RELU, "gelu": esc.ESC_ACT_GELU}[case["act"]]
    if op == "linear":
        esc.esc_linear_forward(s["x"], s["weight"], s["bias"], act, s["out"], s["residual"], s["z"])
        return {k: s[k] for k in ("out", "z") if s[k] is not None}
    if not s["scratch"]:
        s["scratch"]["ws"] = esc.new_linear_workspace(case["rows"], case["K"], case["N"], act, s["x"].dtype)
    esc.esc_linear_backward(s["x"], s["weight"], s["z"], act, s["go"], s["g_x"], s["g_weight"], s["g_bias"], s["scratch"]["ws"])
    return {k: s[k] for k in ("g_x", "g_weight", "g_bias")}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------


def work(case):
    es, rows, op = (4 if case["dtype"] == "fp32" else 2), case["rows"], case["op"]
    if op == "norm":
        return {"bytes": (2 * rows + 2) * case["C"] * es, "flops": 8 * rows * case["C"]}
    if op == "norm_grad":
        return {"bytes": ((4 if case["skip"] else 3) * rows + 3) * case["C"] * es, "flops": 18 * rows * case["C"]}
    K, N = case["K"], case["N"]
    if op == "linear":
        return {"bytes": (rows * (K + N * (1 + case["residual"] + case["keep"])) + N * K + N) * es, "flops": 2 * rows * K * N}
    # read grad_out, z, x and the weights; write their gradients
    return {"bytes": (rows * (2 * K + N * (1 if case["act"] == "none" else 2)) + 2 * N * K + N) * es, "flops": 4 * rows * K * N}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    wide = {k: t.double() for k, t in s.items() if isinstance(t, torch.Tensor)}
    if case["op"] == "norm":
        var, mean = torch.var_mean(wide["x"], 1, unbiased=False, keepdim=True)
        return torch.addcmul(wide["bias"], (wide["x"] - mean) / torch.sqrt(var + EPS), wide["weight"])
    if case["op"] == "norm_grad":
        return _exact_norm_grad(wide)
    if case["op"] == "linear":
        z = torch.addmm(wide["bias"], wide["x"], wide["weight"].T)
        out = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.ndtr(z)}[case["act"]]()
        if "residual" in wide:
            out = out + wide["residual"]
        return {"out": out, "z": z} if "z" in wide else {"out": out}
    g = wide["go"]
    if case["act"] == "relu":
        g = torch.where(wide["z"] > 0, g, torch.zeros_like(g))
    if case["act"] == "gelu":
        z = wide["z"]
        g = g * (torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi))
    return {"g_x": torch.matmul(g, wide["weight"]), "g_weight": torch.einsum("mn,mk->nk", g, wide["x"]), "g_bias": torch.sum(g, 0)}


def _exact_norm_grad(w):
    """The Jacobian of the norm applied to weight * grad_y, term by term."""
    x, a, n = w["x"], w["gy"] * w["weight"], w["x"].shape[1]
    centred = x - x.sum(1, keepdim=True) / n
    spread = torch.sqrt(torch.einsum("rc,rc->r", centred, centred)[:, None] / n + EPS)
    along = torch.einsum("rc,rc->r", a, centred)[:, None]
    g_x = a / spread - a.sum(1, keepdim=True) / (n * spread) - centred * along / (n * spread ** 3)
    if "skip" in w:
        g_x = g_x + w["skip"]
    return {"g_x": g_x, "g_weight": torch.einsum("rc,rc->c", w["gy"], centred / spread), "g_bias": torch.einsum("rc->c", w["gy"])}
