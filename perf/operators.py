"""The operators that train and run the window self-attention of an ESC block, as cases that can be timed and compared.

An ESC block has, beside its ConvAttn modules, one self-attention over non-overlapping windows with a learned relative
position bias, and all of it is trained with AdamW.  The operators here are that attention (forward, and forward with
backward), the bias as a matrix of its own with the gradient of its table, and the optimiser's step over all tensors.

  attention   per window and head: P = softmax(scale q k^T + bias), out = P v; a window at the right or lower border of the
              map holds the pixels that the map has there; bias[i, j] = table[bucket[dy, dx], head] for the offset
              (dy, dx) of query i from key j
  bias        bias[head, i, j] for one window, and the gradient of the table: sums of grad_bias over equal buckets
  adamw       m, v, p of AdamW with decoupled decay over a list of tensors; states in fp32, or m and r = sqrt(v) in e4m3
              with an fp32 scale for each 256 values of a tensor

Keys of a case: op ("forward", "train", "bias", "bias_grad", "adamw"); for the attention dtype, B, H, W, heads, d and the
window wh, ww; for the buckets "offset" (one for every offset), "log" (by sign and logarithm of dy and dx) or "causal" (by
logarithm of the distance back; table is -inf ahead); for adamw the tensors' number and total, the gradients' and the states'
types and whether a bf16 copy of the parameters is kept for the forward pass.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
QUANT = 256            # values of a tensor that share a scale
E4M3_MAX = 448.0
E4M3_LEAST = 2.0 ** -9


def _attention(name, op, dtype, B, H, W, heads, d, wh, ww, buckets="offset"):
    return {"name": name, "op": op, "dtype": dtype, "B": B, "H": H, "W": W, "heads": heads, "d": d, "wh": wh, "ww": ww, "buckets": buckets}


def _bias(name, op, dtype, heads, wh, ww, buckets="offset"):
    return {"name": name, "op": op, "dtype": dtype, "heads": heads, "wh": wh, "ww": ww, "buckets": buckets}


def _adamw(name, tensors, total, grads, states, copy):
    return {"name": name, "op": "adamw", "tensors": tensors, "total": total, "grads": grads, "states": states, "copy": copy}


def listed():
    return [
        # one small crop: latency of a single call (a preview, an interactive crop)
        _attention("att_crop_bf16_64x64", "forward", "bf16", 1, 64, 64, 4, 16, 32, 32),
        # ESC's block on the LR map of x2 super-resolution to 1280x720; 360 rows leave a last row of windows of 8
        _attention("att_x2_bf16_640x360", "forward", "bf16", 1, 360, 640, 4, 16, 32, 32),
        # x3: an odd width, windows of 24, in the precision the paper times
        _attention("att_x3_fp32_427x240", "forward", "fp32", 1, 240, 427, 4, 16, 24, 24),
        # the large model: 192 channels, windows of 48, on the LR map of x4; bias by logarithmic buckets
        _attention("att_large_bf16_320x180", "forward", "bf16", 1, 180, 320, 6, 32, 48, 48, "log"),
        # training: 64 patches of 64x64, forward and backward
        _attention("train_bf16_64x64x64", "train", "bf16", 64, 64, 64, 4, 16, 32, 32),
        # fine-tuning in fp32 at the small width: patches that windows of 24 do not divide
        _attention("train_fp32_4x64x64", "train", "fp32", 4, 64, 64, 3, 16, 24, 24),
        # the bias of the large model's windows as a matrix, for an attention that takes one
        _bias("bias_bf16_6x48x48", "bias", "bf16", 6, 48, 48),
        # its table's gradient for ESC's windows
        _bias("bias_grad_fp32_4x32x32", "bias_grad", "fp32", 4, 32, 32),
        # a sequence instead of a window: 2000 places in one row, logarithmic buckets
        _bias("bias_grad_bf16_2x1x2000_log", "bias_grad", "bf16", 2, 1, 2000, "log"),
        # ESC's parameters: under a million in many small tensors
        _adamw("adamw_esc_fp32", 420, 947_000, "fp32", "fp32", False),
        # a model of 100 million with mixed precision: bf16 gradients, a bf16 copy of the parameters
        _adamw("adamw_100m_bf16_grads", 300, 100_000_000, "bf16", "fp32", True),
        # the same with states in 8 bits
        _adamw("adamw_100m_8bit", 300, 100_000_000, "fp32", "e4m3", False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "train", "train", "bias", "bias_grad", "adamw", "adamw"])
    if op == "adamw":
        tensors = _log_int(rng, 1, 600)
        total = max(tensors, _log_int(rng, 1_000, 100_000_000))
        c = _adamw("", tensors, total, rng.choice(["fp32", "bf16"]), rng.choice(["fp32", "e4m3"]), rng.random() < 0.5)
    else:
        dtype, heads = rng.choice(["bf16", "bf16", "fp32"]), rng.randint(1, 8)
        row = rng.random() < 0.25                                       # a sequence: maps and windows of one row
        buckets = rng.choice(["offset", "log", "causal"]) if row else rng.choice(["offset", "log"])
        wh, ww = (1, _log_int(rng, 1, 2000)) if row else (rng.randint(2, 48), rng.randint(2, 48))
        if op in ("bias", "bias_grad"):
            c = _bias("", op, dtype, heads, wh, ww, buckets)
        else:
            d = rng.choice([8, 10, 16, 16, 24, 30, 32, 32, 48, 64])
            most = (2e8 if op == "forward" else 4e7) if dtype == "fp32" else 8e8   # pairs of one query and one key, by 16 channels
            pixels, B = _log_int(rng, 1, 250_000), rng.choice([1, 1, 2, 3])
            W = pixels if row else max(1, min(pixels, int(math.sqrt(pixels) * rng.uniform(0.6, 1.7))))
            H = 1 if row else max(1, pixels // W)
            while -(-H // wh) * -(-W // ww) * (wh * ww) ** 2 * B * heads * max(1.0, d / 16) > most and (H > 1 or W > 1 or B > 1 or heads > 1):
                if B > 1 or H * W == 1:
                    B, heads = max(1, B - 1), heads if B > 1 else heads - 1
                elif W >= H:
                    W = max(1, W * 2 // 3)
                else:
                    H = max(1, H * 2 // 3)
            c = _attention("", op, dtype, B, H, W, heads, d, wh, ww, buckets)
    del c["name"]
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _log_bucket(v, half, least, most):
    """Sign and logarithm of a distance: distances below `least` have a bucket each, those up to `most` share the rest of `half`."""
    a = v.abs()
    far = least + (torch.log(a.double().clamp(min=1) / least) / math.log(most / least) * (half - least)).long()
    return torch.where(a < least, a, far.clamp(max=half - 1)) + half * (v > 0)


def _buckets(case):
    """(int32 bucket of every offset [2 wh - 1, 2 ww - 1], or None for one bucket each; number of buckets)."""
    wh, ww = case["wh"], case["ww"]
    if case["buckets"] == "offset":
        return None, (2 * wh - 1) * (2 * ww - 1)
    dy = torch.arange(-(wh - 1), wh, device="cuda")[:, None]
    dx = torch.arange(-(ww - 1), ww, device="cuda")[None, :]
    if case["buckets"] == "causal":                                     # the last bucket: keys ahead of the query
        back = _log_bucket(-dx.clamp(min=0), 32, 16, 1024)
        return torch.where(dx < 0, 32, back).to(torch.int32).expand(2 * wh - 1, 2 * ww - 1).contiguous(), 33
    by, bx = _log_bucket(dy, 8, 4, 48), _log_bucket(dx, 16, 8, 512)
    return (by * 32 + bx).to(torch.int32).contiguous(), 16 * 32


def _table(case, n, g, dtype):
    t = torch.randn(n, case["heads"], generator=g, device="cuda") * 0.5
    if case["buckets"] == "causal":
        t[32] = -math.inf
    return t.to(dtype)


def _sizes(case):
    """Sizes of a network's tensors, the same for every seed: a few large ones, many small ones and odd ones, of `total` values together."""
    g = torch.Generator().manual_seed(case["tensors"])
    n, total = case["tensors"], case["total"]
    w = torch.exp(torch.rand(n, generator=g, dtype=torch.float64) * math.log(2000.0))
    sizes = [max(1, int(x)) for x in (w / w.sum() * (total - n)).tolist()]
    sizes[0] += max(0, total - sum(sizes))
    return sizes


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "adamw":
        return _prepare_adamw(case, g)
    dtype = DTYPES[case["dtype"]]
    bucket, n = _buckets(case)
    s = {"case": case, "bucket": bucket, "n": n}
    heads, tokens = case["heads"], case["wh"] * case["ww"]
    if case["op"] == "bias":
        s["table"] = _table(case, n, g, dtype)
        s["bias"] = torch.empty(heads, tokens, tokens, dtype=dtype, device="cuda")
        return s
    if case["op"] == "bias_grad":
        s["grad_bias"] = torch.randn(heads, tokens, tokens, generator=g, device="cuda").to(dtype)
        s["g_table"] = torch.empty(n, heads, device="cuda")
        s["scratch"] = {}
        return s
    B, H, W, C = case["B"], case["H"], case["W"], heads * case["d"]
    # one projection gives q, k and v of a pixel side by side
    s["qkv"] = torch.randn(B, H, W, 3 * C, generator=g, device="cuda").to(dtype)
    s["table"] = _table(case, n, g, dtype)
    s["scale"] = case["d"] ** -0.5
    s["out"] = torch.empty(B, H, W, C, dtype=dtype, device="cuda")
    if case["op"] == "train":
        s["go"] = torch.randn(B, H, W, C, generator=g, device="cuda").to(dtype)
        s["lse"] = torch.empty(B, heads, H, W, device="cuda")
        s["g_qkv"] = torch.empty_like(s["qkv"])
        s["g_table"] = torch.empty_like(s["table"])
        s["scratch"] = {}
    return s


def _prepare_adamw(case, g):
    sizes = _sizes(case)
    starts, at = [], 0
    for n in sizes:                                                     # every tensor starts at a scale's border, as an allocation would
        starts.append(at)
        at += -(-n // QUANT) * QUANT
    edge = torch.zeros(at + 1, dtype=torch.int32, device="cuda")
    first = torch.tensor(starts, device="cuda")
    edge[first] += 1
    edge.index_add_(0, first + torch.tensor(sizes, device="cuda"), torch.full((len(sizes),), -1, dtype=torch.int32, device="cuda"))
    real = edge.cumsum(0)[:at] > 0
    of = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor([-(-n // QUANT) * QUANT for n in sizes], device="cuda"), output_size=at)
    # gradients of a layer have a scale of their own
    spread = torch.exp(torch.randn(len(sizes), generator=g, device="cuda") * 2 - 7)[of]
    s = {"case": case, "sizes": sizes, "starts": starts, "real": real, "step": 100,
         "lr": 5e-4, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "decay": 0.01, "grad_scale": 0.5}
    s["p"] = torch.randn(at, generator=g, device="cuda") * 0.05 * real
    s["g"] = (torch.randn(at, generator=g, device="cuda") * spread * real).to(DTYPES[case["grads"]])
    m = torch.randn(at, generator=g, device="cuda") * spread * 0.1 * real
    r = torch.exp(torch.randn(at, generator=g, device="cuda") * 0.5) * spread * 0.5 * real
    del spread, of
    if case["states"] == "e4m3":
        s["m"], s["m_scale"] = _pack(m, False)
        s["r"], s["r_scale"] = _pack(r, True)
    else:
        s["m"], s["v"] = m, r * r
    s["copy"] = torch.zeros(at, dtype=torch.bfloat16, device="cuda") if case["copy"] else None
    s["plan"] = None
    return s


# ---- the operators' plain forms ---------------------------------------------------------------------------------------------


def _index(case, bucket):
    """Bucket of every (query, key) of one window, int64 [tokens, tokens]."""
    wh, ww = case["wh"], case["ww"]
    t = torch.arange(wh * ww, device="cuda")
    y, x = t // ww, t % ww
    at = (y[:, None] - y[None] + wh - 1) * (2 * ww - 1) + (x[:, None] - x[None] + ww - 1)
    return at if bucket is None else bucket.reshape(-1)[at].long()


def _windows(t, case, heads):
    """[B, H, W, heads * d] -> [windows, heads, tokens, d] in 32 bits, with zeros where the map has no pixels."""
    B, H, W, C = t.shape
    wh, ww = case["wh"], case["ww"]
    ny, nx = -(-H // wh), -(-W // ww)
    p = torch.zeros(B, ny * wh, nx * ww, C, device="cuda")
    p[:, :H, :W] = t
    return p.view(B, ny, wh, nx, ww, heads, C // heads).permute(0, 1, 3, 5, 2, 4, 6).reshape(B * ny * nx, heads, wh * ww, C // heads)


def _map(w, case, dtype):
    """The inverse of _windows, rounded once."""
    B, H, W, wh, ww = case["B"], case["H"], case["W"], case["wh"], case["ww"]
    ny, nx, heads, d = -(-H // wh), -(-W // ww), w.shape[1], w.shape[3]
    p = w.view(B, ny, nx, heads, wh, ww, d).permute(0, 1, 4, 2, 5, 3, 6).reshape(B, ny * wh, nx * ww, heads * d)
    return p[:, :H, :W].to(dtype)


def _plain_attention(s):
    case, qkv = s["case"], s["qkv"]
    heads, C, dtype = case["heads"], case["heads"] * case["d"], qkv.dtype
    q, k, v = (_windows(qkv[..., i * C:(i + 1) * C], case, heads) for i in range(3))
    inside = _windows(torch.ones(case["B"], case["H"], case["W"], 1, device="cuda"), case, 1)[:, :, :, 0]
    index = _index(case, s["bucket"])
    x = (q @ k.transpose(2, 3)) * s["scale"]
    x += s["table"].float().t()[:, index]
    x.masked_fill_(inside[:, :, None, :] == 0, -math.inf)
    top = x.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = x.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    p /= torch.where(total == 0, 1.0, total)
    out = p @ v
    if case["op"] == "forward":
        return _map(out, case, dtype)
    lse = torch.where(total == 0, -math.inf, total.log() + top)
    go = _windows(s["go"], case, heads)
    g_v = p.transpose(2, 3) @ go
    ds = go @ v.transpose(2, 3)
    ds -= (go * out).sum(3, keepdim=True)
    ds *= p
    ds *= inside[:, :, :, None]
    g_q, g_k = (ds @ k) * s["scale"], (ds.transpose(2, 3) @ q) * s["scale"]
    by_pair = ds.sum(0, dtype=torch.float64)
    g_table = torch.zeros(s["n"], heads, dtype=torch.float64, device="cuda")
    g_table.index_add_(0, index.reshape(-1), by_pair.reshape(heads, -1).t().contiguous())
    return {"out": _map(out, case, dtype), "lse": _map(lse, case, torch.float32).permute(0, 3, 1, 2),
            "g_qkv": torch.cat([_map(t, case, dtype) for t in (g_q, g_k, g_v)], 3), "g_table": g_table.to(dtype)}


def _plain_bias(s):
    return s["table"].t()[:, _index(s["case"], s["bucket"])]


def _plain_bias_grad(s):
    g_table = torch.zeros(s["n"], s["case"]["heads"], dtype=torch.float64, device="cuda")
    g = s["grad_bias"].double()
    g_table.index_add_(0, _index(s["case"], s["bucket"]).reshape(-1), g.reshape(g.shape[0], -1).t().contiguous())
    return g_table.float()


def _pack(t, root):
    """e4m3 values and the fp32 scale of each 256 of them; a root that is not zero stays so."""
    b = t.view(-1, QUANT)
    top = b.abs().amax(1, keepdim=True)
    some = top >= 1e-30
    inverse = torch.where(some, E4M3_MAX / torch.where(some, top, 1.0), 0.0)
    scale = torch.where(some, top / E4M3_MAX, 0.0)
    x = b * inverse
    if root:
        x = torch.where((b > 0) & (x < E4M3_LEAST) & some, E4M3_LEAST, x)
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(-1), scale.view(-1)


def _held(codes, scale):
    return (codes.float().view(-1, QUANT) * scale[:, None]).view(-1)


def _plain_adamw(s):
    """Every operation is rounded to 32 bits as it stands, so that what is held in 8 bits falls to the same side everywhere."""
    eight = s["case"]["states"] == "e4m3"
    t = s["step"]
    b1, b2, one1, one2 = s["beta1"], s["beta2"], 1 - s["beta1"], 1 - s["beta2"]
    size, root = s["lr"] / (1 - b1 ** t), 1 / math.sqrt(1 - b2 ** t)
    g = s["g"].float() * s["grad_scale"]
    m = _held(s["m"], s["m_scale"]) if eight else s["m"]
    v = _held(s["r"], s["r_scale"]).square() if eight else s["v"]
    m = m * b1 + g * one1
    v = v * b2 + g * g * one2
    r = v.sqrt()
    s["p"].mul_(1 - s["lr"] * s["decay"]).sub_(m / (r * root + s["eps"]) * size)
    if s["copy"] is not None:
        s["copy"].copy_(s["p"])
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return
    for name, x, scale in (("m", m, "m_scale"), ("r", r, "r_scale")):
        codes, scales = _pack(x, name == "r")
        s[name].copy_(codes)
        s[scale].copy_(scales)


def _adamw_outputs(s):
    got = {"p": s["p"], "copy": s["copy"]}
    if s["case"]["states"] == "e4m3":
        got |= {"m": _held(s["m"], s["m_scale"]), "r": _held(s["r"], s["r_scale"]), "m_scale": s["m_scale"], "r_scale": s["r_scale"]}
    else:
        got |= {"m": s["m"], "v": s["v"]}
    return {k: x for k, x in got.items() if x is not None}


# ---- one pass ---------------------------------------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(state, op)
    if op == "adamw":
        state["step"] += 1
        _plain_adamw(state)
        return _adamw_outputs(state)
    if op == "bias":
        return _plain_bias(state)
    if op == "bias_grad":
        return _plain_bias_grad(state)
    return _plain_attention(state)


def _run_own(s, op):
    import paper_2503_06671_b200 as esc

    case = s["case"]
    if op == "adamw":
        if s["plan"] is None:                                           # once for the tensors' addresses, as a program does
            eight = case["states"] == "e4m3"
            at, sizes = s["starts"], s["sizes"]
            cut = lambda t: [t[a:a + n] for a, n in zip(at, sizes)]     # noqa: E731
            scales = lambda t: [t[a // QUANT:a // QUANT - (-n // QUANT)] for a, n in zip(at, sizes)]   # noqa: E731
            s["plan"] = esc.new_adamw_plan(cut(s["p"]), cut(s["g"]), cut(s["m"]), cut(s["r"] if eight else s["v"]),
                                           scales(s["m_scale"]) if eight else None, scales(s["r_scale"]) if eight else None,
                                           cut(s["copy"]) if s["copy"] is not None else None)
        s["step"] += 1
        esc.esc_adamw_step(s["plan"], s["step"], s["lr"], s["beta1"], s["beta2"], s["eps"], s["decay"], grad_scale=s["grad_scale"])
        return _adamw_outputs(s)
    if op == "bias":
        return esc.esc_relpos_bias_forward(s["table"], s["bucket"], case["wh"], case["ww"], s["bias"])
    if op == "bias_grad":
        if not s["scratch"]:
            s["scratch"]["ws"] = esc.new_relpos_bias_workspace(case["heads"], case["wh"], case["ww"])
        return esc.esc_relpos_bias_backward(s["grad_bias"], s["bucket"], case["wh"], case["ww"], s["g_table"], s["scratch"]["ws"])
    C = case["heads"] * case["d"]
    q, k, v = s["qkv"][..., :C], s["qkv"][..., C:2 * C], s["qkv"][..., 2 * C:]
    if op == "forward":
        return esc.esc_window_attention_forward(q, k, v, case["heads"], case["wh"], case["ww"], s["table"], s["bucket"], s["scale"], s["out"])
    if not s["scratch"]:
        s["scratch"]["ws"] = esc.new_window_attention_workspace(case["B"], case["heads"], case["d"], case["H"], case["W"], case["wh"], case["ww"])
    esc.esc_window_attention_forward(q, k, v, case["heads"], case["wh"], case["ww"], s["table"], s["bucket"], s["scale"], s["out"], s["lse"])
    g = s["g_qkv"]
    esc.esc_window_attention_backward(q, k, v, case["heads"], case["wh"], case["ww"], s["table"], s["bucket"], s["scale"], s["out"], s["lse"],
                                      s["go"], g[..., :C], g[..., C:2 * C], g[..., 2 * C:], s["g_table"], s["scratch"]["ws"])
    return {"out": s["out"], "lse": s["lse"], "g_qkv": g, "g_table": s["g_table"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------


def _pairs(case):
    """Pairs of a query and a key over all windows, for one head."""
    def side(n, w):
        return (n // w) * w * w + (n % w) ** 2

    return case["B"] * side(case["H"], case["wh"]) * side(case["W"], case["ww"])


def work(case):
    if case["op"] == "adamw":
        grad = 4 if case["grads"] == "fp32" else 2
        state = 16 if case["states"] == "fp32" else 4 + 4 * 4 / QUANT
        return {"bytes": case["total"] * (8 + grad + state + (2 if case["copy"] else 0)), "flops": case["total"] * 15}
    es, tokens = (4 if case["dtype"] == "fp32" else 2), case["wh"] * case["ww"]
    if case["op"] in ("bias", "bias_grad"):
        return {"bytes": case["heads"] * tokens * tokens * es, "flops": case["heads"] * tokens * tokens if case["op"] == "bias_grad" else 0}
    values = case["B"] * case["H"] * case["W"] * case["heads"] * case["d"]
    pairs = _pairs(case) * case["heads"]
    if case["op"] == "forward":
        return {"bytes": 4 * values * es, "flops": 4 * case["d"] * pairs}
    # read q, k, v and grad_out, write out and three gradients; two products forward, five backward
    return {"bytes": 8 * values * es, "flops": 14 * case["d"] * pairs}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    if case["op"] == "bias":
        return s["table"].double()[_exact_bucket(case, s["bucket"], case["wh"], case["ww"])].permute(2, 0, 1)
    if case["op"] == "bias_grad":
        at = _exact_bucket(case, s["bucket"], case["wh"], case["ww"]).reshape(-1)
        g = torch.zeros(case["heads"], s["n"], dtype=torch.float64, device="cuda")
        for h in range(case["heads"]):
            g[h] = torch.bincount(at, weights=s["grad_bias"][h].double().reshape(-1), minlength=s["n"])
        return g.t().contiguous()
    return _exact_attention(s)


def _exact_bucket(case, bucket, h, w):
    """Bucket of every (query, key) of a window of h x w pixels."""
    y = torch.arange(h, device="cuda").repeat_interleave(w)
    x = torch.arange(w, device="cuda").repeat(h)
    dy, dx = y.unsqueeze(1) - y.unsqueeze(0), x.unsqueeze(1) - x.unsqueeze(0)
    at = (dy + case["wh"] - 1) * (2 * case["ww"] - 1) + dx + case["ww"] - 1
    return at if bucket is None else bucket.flatten().long()[at]


def _exact_attention(s):
    """One window of the map after another, in 64 bits."""
    case = s["case"]
    B, H, W, heads, d, wh, ww = (case[k] for k in ("B", "H", "W", "heads", "d", "wh", "ww"))
    if B * (H / wh + 1) * (W / ww + 1) > 20000:
        return None
    C, train = heads * d, case["op"] == "train"
    out = torch.zeros(B, H, W, C, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, heads, H, W, dtype=torch.float64, device="cuda")
    g_qkv = torch.zeros(B, H, W, 3 * C, dtype=torch.float64, device="cuda") if train else None
    g_table = torch.zeros(heads, s["n"], dtype=torch.float64, device="cuda")
    table = s["table"].double()
    at_of = {}
    few = max(1, int(2e7 // (heads * (min(wh, H) * min(ww, W)) ** 2)))  # images at a time
    for y in range(0, H, wh):
        for x in range(0, W, ww):
            h, w = min(wh, H - y), min(ww, W - x)
            if (h, w) not in at_of:
                at_of[h, w] = _exact_bucket(case, s["bucket"], h, w)
            at = at_of[h, w]
            bias = table[at].permute(2, 0, 1)
            for b in range(0, B, few):
                part = slice(b, min(B, b + few)), slice(y, y + h), slice(x, x + w)
                tokens = s["qkv"][part].double().reshape(-1, h * w, 3, heads, d)
                q, k, v = (tokens[:, :, i].transpose(1, 2) for i in range(3))
                logits = torch.einsum("bhid,bhjd->bhij", q, k) * s["scale"] + bias
                total = torch.logsumexp(logits, 3, keepdim=True)
                p = torch.where(total == -math.inf, torch.zeros_like(logits), torch.exp(logits - total))
                o = torch.einsum("bhij,bhjd->bhid", p, v)
                out[part] = o.transpose(1, 2).reshape(-1, h, w, C)
                if not train:
                    continue
                lse[part[0], :, part[1], part[2]] = total.reshape(-1, heads, h, w)
                go = s["go"][part].double().reshape(-1, h * w, heads, d).transpose(1, 2)
                dp = torch.einsum("bhid,bhjd->bhij", go, v)
                ds = p * (dp - (p * dp).sum(3, keepdim=True))
                grads = [torch.einsum("bhij,bhjd->bhid", ds, k) * s["scale"], torch.einsum("bhij,bhid->bhjd", ds, q) * s["scale"],
                         torch.einsum("bhij,bhid->bhjd", p, go)]
                g_qkv[part] = torch.stack(grads, 3).permute(0, 2, 3, 1, 4).reshape(-1, h, w, 3 * C)
                for n in range(heads):
                    g_table[n] += torch.bincount(at.reshape(-1), weights=ds[:, n].sum(0).reshape(-1), minlength=s["n"])
    return {"out": out, "lse": lse, "g_qkv": g_qkv, "g_table": g_table.t().contiguous()} if train else out


def _exact_adamw(s):
    """What is held in 8 bits has no value in 64 (a code is a choice between neighbours that 32 bits make); the scales have."""
    eight = s["case"]["states"] == "e4m3"
    t = s["step"] + 1
    g = s["g"].double() * s["grad_scale"]
    if eight:
        widen = lambda c, k: c.double() * k.double().repeat_interleave(QUANT)   # noqa: E731
        m, v = widen(s["m"], s["m_scale"]), widen(s["r"], s["r_scale"]) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m = s["beta1"] * m + (1 - s["beta1"]) * g
    v = s["beta2"] * v + (1 - s["beta2"]) * g ** 2
    del g
    step = s["lr"] * (m / (1 - s["beta1"] ** t)) / (torch.sqrt(v / (1 - s["beta2"] ** t)) + s["eps"])
    p = s["p"].double() * (1 - s["lr"] * s["decay"]) - step
    got = {"p": p, "copy": p if s["copy"] is not None else None}
    if eight:
        top = lambda x: x.abs().reshape(-1, QUANT).amax(1) / E4M3_MAX   # noqa: E731
        return got | {"m": None, "r": None, "m_scale": top(m), "r_scale": top(torch.sqrt(v))}
    return got | {"m": m, "v": v}
