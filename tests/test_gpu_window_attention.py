"""The window self-attention (ESC Section 3.3) forward and backward against the formulas in 64 bits, element by element, within the
bounds of attention_ref: sizes from one pixel to many windows, odd widths, borders, every width of a head, packed and other strides,
buckets, masks that leave rows empty; captured graphs, streams, two calls at once."""
import math

import numpy as np
import pytest
import torch

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


SHAPES = [
    # B, H, W, heads, d, wh, ww
    (1, 1, 1, 1, 16, 1, 1),          # one pixel
    (2, 3, 5, 1, 8, 3, 5),           # one small window per image
    (1, 5, 7, 3, 16, 8, 8),          # a map smaller than its window
    (1, 16, 16, 4, 16, 8, 8),
    (2, 33, 47, 2, 16, 16, 16),      # borders of one row and of 15 columns
    (1, 24, 50, 3, 16, 24, 24),      # windows that no power of two divides
    (1, 20, 31, 2, 10, 7, 9),        # odd windows, a head of 10 channels
    (1, 32, 64, 2, 16, 32, 32),
    (1, 40, 33, 1, 16, 32, 32),      # borders of 8 rows and of one column
    (1, 18, 22, 2, 30, 12, 12),
    (1, 17, 26, 2, 32, 16, 13),
    (1, 30, 30, 1, 24, 15, 30),
    (1, 19, 23, 2, 48, 10, 12),
    (2, 13, 11, 2, 64, 8, 6),
    (1, 50, 50, 1, 32, 48, 48),      # the large model's windows
    (1, 1, 1, 2, 16, 1, 300),        # a sequence of one
    (2, 1, 129, 2, 32, 1, 129),
    (1, 1, 700, 1, 16, 1, 333),      # two whole windows and a rest of 34
    (1, 9, 3, 2, 1, 4, 2),           # one channel
    (1, 6, 6, 9, 3, 3, 3),           # many narrow heads: nothing is aligned
    (1, 40, 66, 1, 64, 64, 64),      # the largest square window: little shared memory is left beside its table
    (1, 1, 900, 1, 16, 1, 8192),     # the longest sequence's table
    (1, 3, 37, 2, 20, 64, 2),        # tall narrow windows
]


def inputs(shape, dtype, seed, buckets="offset", spread=1.0):
    B, H, W, heads, d, wh, ww = shape
    g = torch.Generator().manual_seed(seed)
    t = DTYPES[dtype]
    C = heads * d
    x = {n: (torch.randn(B, H, W, C, generator=g) * spread).to(t) for n in ("q", "k", "v", "go")}
    offsets = (2 * wh - 1) * (2 * ww - 1)
    bucket = None if buckets == "offset" else torch.randint(0, 11, (offsets,), generator=g, dtype=torch.int32)
    x["table"] = torch.randn(offsets if bucket is None else 11, heads, generator=g).to(t)
    x["bucket"] = bucket
    return x


def run(pkg, x, shape, scale, packed=True, pad=0, backward=True):
    """The two calls on the device; q, k, v and their gradients as slices of packed tensors, or each with `pad` values between pixels."""
    B, H, W, heads, d, wh, ww = shape
    C = heads * d
    dev = {n: x[n].cuda() if x[n] is not None else None for n in ("table", "bucket", "go")}
    if packed:
        qkv = torch.cat([x[n] for n in "qkv"], 3).cuda()
        q, k, v = (qkv[..., i * C:(i + 1) * C] for i in range(3))
        g = torch.full_like(qkv, 7.0)
        gq, gk, gv = (g[..., i * C:(i + 1) * C] for i in range(3))
    else:
        wide = [torch.full((B, H, W, C + pad), 5.0, dtype=x["q"].dtype, device="cuda") for _ in range(6)]
        for t, n in zip(wide, "qkv"):
            t[..., :C] = x[n].cuda()
        q, k, v, gq, gk, gv = (t[..., :C] for t in wide)
    out = torch.full((B, H, W, C), float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full((B, heads, H, W), float("nan"), device="cuda")
    pkg.esc_window_attention_forward(q, k, v, heads, wh, ww, dev["table"], dev["bucket"], scale, out, lse)
    got = {"out": out, "lse": lse}
    if backward:
        gt = torch.full_like(dev["table"], 3.0) if dev["table"] is not None else None
        ws = pkg.new_window_attention_workspace(B, heads, d, H, W, wh, ww)
        ws.fill_(0xFF)                                                   # NaN: nothing may be read before it is written
        pkg.esc_window_attention_backward(q, k, v, heads, wh, ww, dev["table"], dev["bucket"], scale, out, lse, dev["go"], gq, gk, gv, gt, ws)
        got |= {"g_q": gq, "g_k": gk, "g_v": gv, "g_table": gt}
    torch.cuda.synchronize()
    if not packed and pad:
        for t in wide:
            assert (t[..., C:] == 5.0).all(), "values between the pixels were written"
    return got


def compare(got, x, shape, scale, dtype):
    heads, wh, ww = shape[3], shape[5], shape[6]
    val, far = ref.attention(x["q"], x["k"], x["v"], heads, wh, ww, x["table"], x["bucket"], scale, x["go"] if "g_q" in got else None, dtype == "bf16")
    for n, t in got.items():
        if t is not None:
            ref.check(t, val[n], far[n], n)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_attention(pkg, shape, dtype):
    x = inputs(shape, dtype, sum(shape))
    compare(run(pkg, x, shape, shape[4] ** -0.5), x, shape, shape[4] ** -0.5, dtype)


def test_many_windows_of_one_block(pkg):
    """More windows than a block of the table's gradient lists at a time, whole ones and cut ones: 300 heads leave a block all of them."""
    shape = (1, 8 * 15 + 3, 8 * 10 + 5, 300, 2, 8, 8)
    x = inputs(shape, "bf16", 21)
    compare(run(pkg, x, shape, 0.7), x, shape, 0.7, "bf16")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_own_tensors_and_strides(pkg, dtype, pad):
    shape = (2, 13, 21, 2, 16, 8, 12)
    x = inputs(shape, dtype, 5 + pad, "some")
    compare(run(pkg, x, shape, 0.3, packed=False, pad=pad), x, shape, 0.3, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_unaligned_pointers(pkg, dtype):
    """q, k, v start in the middle of a 16-byte piece."""
    shape = (1, 9, 10, 2, 16, 6, 5)
    B, H, W, heads, d, wh, ww = shape
    x = inputs(shape, dtype, 8)
    C = heads * d
    wide = {n: torch.zeros(B, H, W, C + 3, dtype=DTYPES[dtype], device="cuda") for n in "qkv"}
    for n in "qkv":
        wide[n][..., 1:C + 1] = x[n].cuda()
    out, lse = torch.empty(B, H, W, C, dtype=DTYPES[dtype], device="cuda"), torch.empty(B, heads, H, W, device="cuda")
    pkg.esc_window_attention_forward(*(wide[n][..., 1:C + 1] for n in "qkv"), heads, wh, ww, x["table"].cuda(), None, 0.25, out, lse)
    compare({"out": out, "lse": lse}, x, shape, 0.25, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_bias(pkg, dtype):
    shape = (1, 20, 20, 2, 16, 10, 10)
    x = inputs(shape, dtype, 9) | {"table": None}
    compare(run(pkg, x, shape, 0.25), x, shape, 0.25, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_gradient_of_the_table_and_two_streams(pkg, dtype):
    """Without grad_table the others are the same bits; two backward calls at once on two streams, each with its workspace."""
    shape = (2, 30, 40, 2, 16, 12, 16)
    B, H, W, heads, d, wh, ww = shape
    x = inputs(shape, dtype, 30)
    want = run(pkg, x, shape, 0.25)
    q, k, v, go, table = (x[n].cuda() for n in ("q", "k", "v", "go", "table"))
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            g = [torch.full_like(q, 7.0) for _ in range(3)]
            gt = torch.full_like(table, 7.0) if i else None
            out, lse = torch.empty_like(q), torch.empty(B, heads, H, W, device="cuda")
            for _ in range(3):
                pkg.esc_window_attention_forward(q, k, v, heads, wh, ww, table, None, 0.25, out, lse)
                pkg.esc_window_attention_backward(q, k, v, heads, wh, ww, table, None, 0.25, out, lse, go, *g, gt)
            got.append((out, lse, *g, gt))
    torch.cuda.synchronize()
    for r in got:
        for n, t in zip(("out", "lse", "g_q", "g_k", "g_v", "g_table"), r):
            assert t is None or torch.equal(t.contiguous(), want[n].contiguous()), n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mask", ["inf", "lowest", "-10000"])
@pytest.mark.parametrize("kind", ["ahead", "all", "some rows"])
def test_masks(pkg, dtype, kind, mask):
    """Masked: keys ahead of the query, every key, all keys of some queries; by -inf, the type's lowest value and -10000, which are one."""
    shape = (1, 1, 150, 2, 16, 1, 75)
    x = inputs(shape, dtype, 10)
    dx = torch.arange(-74, 75)
    off = {"ahead": dx < 0, "all": dx < 99, "some rows": dx > -20}[kind]   # the last: only keys at least 20 ahead, so the last 20 queries have none
    x["table"][off] = {"inf": -math.inf, "lowest": torch.finfo(DTYPES[dtype]).min, "-10000": -10000.0}[mask]
    got = run(pkg, x, shape, 0.25)
    x["table"][off] = -math.inf
    compare(got, x, shape, 0.25, dtype)
    if kind == "all":
        assert (got["out"] == 0).all() and (got["lse"] == -math.inf).all()
        assert all((got[n] == 0).all() for n in ("g_q", "g_k", "g_v", "g_table"))


@pytest.mark.parametrize("dtype", DTYPES)
def test_buckets_outside_the_table(pkg, dtype):
    shape = (1, 12, 12, 2, 16, 6, 6)
    x = inputs(shape, dtype, 11, "some")
    x["bucket"][::3] = -1
    x["bucket"][1::5] = 2 ** 31 - 1
    compare(run(pkg, x, shape, 0.25), x, shape, 0.25, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores(pkg, dtype):
    """Rows that one key dominates, far from zero: the running maximum has to move."""
    shape = (1, 16, 40, 1, 16, 16, 20)
    x = inputs(shape, dtype, 12, spread=4.0)
    x["table"] = x["table"] * 20
    compare(run(pkg, x, shape, 1.0), x, shape, 1.0, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_same_bits_again(pkg, dtype):
    shape = (3, 40, 40, 2, 16, 16, 16)
    x = inputs(shape, dtype, 13, "some")
    a, b = run(pkg, x, shape, 0.25), run(pkg, x, shape, 0.25)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dtype", DTYPES)
def test_windows_do_not_see_each_other(pkg, dtype):
    """NaN in one window leaves the others' results alone (its own rows and keys, and the shared table's gradient, are lost)."""
    shape = (1, 16, 24, 2, 16, 8, 8)
    x = inputs(shape, dtype, 14)
    a = run(pkg, x, shape, 0.25)
    x["q"][0, 3, 9] = math.nan
    x["k"][0, 4, 10] = math.inf
    b = run(pkg, x, shape, 0.25)
    keep = torch.ones(16, 24, dtype=torch.bool)
    keep[:8, 8:16] = False
    for n in ("out", "g_q", "g_k", "g_v"):
        assert torch.equal(a[n][0][keep], b[n][0][keep]), n


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_and_replayed(pkg, dtype):
    """Forward and backward in one graph on a side stream, replayed on new inputs, beside an eager call of another workspace."""
    shape = (2, 24, 40, 2, 16, 16, 16)
    B, H, W, heads, d, wh, ww = shape
    C = heads * d
    x, y = inputs(shape, dtype, 15), inputs(shape, dtype, 16)
    stream = torch.cuda.Stream()
    t = {n: x[n].cuda() for n in ("q", "k", "v", "go", "table")}
    got = {n: torch.zeros_like(t[m]) for n, m in (("out", "q"), ("g_q", "q"), ("g_k", "q"), ("g_v", "q"), ("g_table", "table"))}
    got["lse"] = torch.zeros(B, heads, H, W, device="cuda")
    ws = pkg.new_window_attention_workspace(B, heads, d, H, W, wh, ww)
    torch.cuda.synchronize()

    def both():
        pkg.esc_window_attention_forward(t["q"], t["k"], t["v"], heads, wh, ww, t["table"], None, 0.25, got["out"], got["lse"])
        pkg.esc_window_attention_backward(t["q"], t["k"], t["v"], heads, wh, ww, t["table"], None, 0.25, got["out"], got["lse"], t["go"],
                                          got["g_q"], got["g_k"], got["g_v"], got["g_table"], ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        both()
    for n in t:
        t[n].copy_(y[n])
    torch.cuda.synchronize()
    graph.replay()
    other = run(pkg, x, shape, 0.25)                                     # its own tensors and workspace, at the same time
    torch.cuda.synchronize()
    compare(got, y, shape, 0.25, dtype)
    compare(other, x, shape, 0.25, dtype)


def test_gradients_against_differences(pkg):
    """Along a random direction in q, k, v and the table: the fp32 kernel's gradients against central differences of the formula in 64
    bits (their own error: 1e-4^2 of the third derivative, below 1e-6 of the scale here)."""
    shape = (1, 9, 14, 2, 16, 6, 7)
    B, H, W, heads, d, wh, ww = shape
    x = inputs(shape, "fp32", 17, "some")
    got = run(pkg, x, shape, 0.25)
    g = torch.Generator().manual_seed(3)
    to = {n: torch.randn(x[n].shape, generator=g, dtype=torch.float64) for n in ("q", "k", "v", "table")}

    def loss(e):
        z = {n: x[n].double() + e * to[n] for n in to}
        val, _ = ref.attention(z["q"], z["k"], z["v"], heads, wh, ww, z["table"], x["bucket"], 0.25)
        return (val["out"] * x["go"].double()).sum().item()

    slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
    names = {"q": "g_q", "k": "g_k", "v": "g_v", "table": "g_table"}
    terms = [got[names[n]].double().cpu() * to[n] for n in to]
    mine, scale = sum(t.sum().item() for t in terms), sum(t.abs().sum().item() for t in terms)
    assert abs(mine - slope) <= 1e-5 * scale, (mine, slope, scale)


def test_long_strides(pkg):
    """Pixels so far apart that offsets pass 32 bits: 2.2e9 values between the first and the last row of the map."""
    heads, d, wh, ww = 1, 16, 2, 2
    H, W, step = 3, 2, 440_000_000
    room = torch.empty(step * (H * W - 1) + 64, dtype=torch.bfloat16, device="cuda")
    x = inputs((1, H, W, heads, d, wh, ww), "bf16", 18)
    at = lambda off: torch.as_strided(room, (1, H, W, heads * d), (H * W * step, W * step, step, 1), off)   # noqa: E731
    q, k, v = at(0), at(16), at(32)
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        t.copy_(x[n].cuda())
    out = torch.empty(1, H, W, heads * d, dtype=torch.bfloat16, device="cuda")
    pkg.esc_window_attention_forward(q, k, v, heads, wh, ww, x["table"].cuda(), None, 0.25, out)
    compare({"out": out}, x, (1, H, W, heads, d, wh, ww), 0.25, "bf16")


def test_binding_refuses(pkg):
    q = torch.zeros(1, 8, 8, 32, device="cuda")
    table, out = torch.zeros(225, 2, device="cuda"), torch.zeros(1, 8, 8, 32, device="cuda")
    ok = lambda **o: pkg.esc_window_attention_forward(*[o.get(n, q) for n in "qkv"], 2, 8, 8, o.get("table", table), o.get("bucket"), 0.25, o.get("out", out))   # noqa: E731
    ok()
    for bad in ({"k": q.bfloat16()}, {"v": q[:, :, :4]}, {"q": q.transpose(1, 2)}, {"out": out[..., :16]}, {"table": table[:, :1]}, {"table": table.bfloat16()},
                {"bucket": torch.zeros(3, dtype=torch.int32, device="cuda")}, {"out": out.cpu()}):
        with pytest.raises(ValueError):
            ok(**bad)
    with pytest.raises(pkg.EscError):
        ok(out=q)                                                        # in place
    with pytest.raises(pkg.EscError):
        ok(table=table[:224].contiguous())                               # a row per offset is needed without buckets
    assert np.isfinite(out.cpu().numpy()).all()
