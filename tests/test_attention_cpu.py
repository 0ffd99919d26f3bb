"""The formulas that the GPU tests hold the window attention to, against automatic differentiation and differences, and what the
entry points refuse on the host, before anything could be launched."""
import ctypes
import math

import pytest
import torch

from tests import attention_ref as ref


@pytest.fixture(scope="module")
def L():
    from paper_2503_06671_b200 import build, lib

    build.build()
    return lib()


@pytest.mark.parametrize("buckets", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 2, 1, 1), (2, 5, 7, 2, 3, 4, 3), (1, 1, 9, 1, 4, 1, 5), (1, 3, 3, 2, 2, 8, 8)])
def test_formulas_against_autograd_and_differences(shape, buckets):
    B, H, W, heads, d, wh, ww = shape
    g = torch.Generator().manual_seed(sum(shape))
    offsets = (2 * wh - 1) * (2 * ww - 1)
    bucket = torch.randint(-1, 4, (offsets,), generator=g) if buckets else None
    x = {n: torch.randn(B, H, W, heads * d, generator=g, dtype=torch.float64, requires_grad=True) for n in "qkv"}
    x["table"] = torch.randn(4 if buckets else offsets, heads, generator=g, dtype=torch.float64, requires_grad=True)
    go = torch.randn(B, H, W, heads * d, generator=g, dtype=torch.float64)

    def out_of(q, k, v, table):
        out = torch.zeros(B, H, W, heads * d, dtype=torch.float64)
        for y in range(H):
            for z in range(W):
                mates = [(a, b) for a in range(H) for b in range(W) if a // wh == y // wh and b // ww == z // ww]
                for h in range(heads):
                    c = slice(h * d, (h + 1) * d)
                    logits = []
                    for a, b in mates:
                        o = (y - a + wh - 1) * (2 * ww - 1) + z - b + ww - 1
                        row = o if bucket is None else int(bucket[o])
                        bias = table[row, h] if 0 <= row < table.shape[0] else torch.zeros((), dtype=torch.float64)
                        logits.append(0.5 * (q[:, y, z, c] * k[:, a, b, c]).sum(1) + bias)
                    p = torch.softmax(torch.stack(logits, 1), 1)
                    o = sum(p[:, i:i + 1] * v[:, a, b, c] for i, (a, b) in enumerate(mates))
                    out = out.index_put((torch.arange(B)[:, None], torch.tensor(y), torch.tensor(z), torch.arange(h * d, (h + 1) * d)[None]), o)
        return out

    want = out_of(*(x[n] for n in ("q", "k", "v", "table")))
    grads = torch.autograd.grad((want * go).sum(), [x[n] for n in ("q", "k", "v", "table")], allow_unused=True)
    val, far = ref.attention(*(x[n].detach() for n in "qkv"), heads, wh, ww, x["table"].detach(), bucket, 0.5, go)
    assert torch.allclose(val["out"], want.detach(), rtol=0, atol=1e-12)
    for n, t in zip(("g_q", "g_k", "g_v", "g_table"), grads):
        assert torch.allclose(val[n], torch.zeros_like(val[n]) if t is None else t, rtol=0, atol=1e-12), n
        assert (far[n] >= 0).all()
    to = {n: torch.randn(x[n].shape, generator=g, dtype=torch.float64) for n in x}
    at = lambda e: (ref.attention(*(x[n].detach() + e * to[n] for n in "qkv"), heads, wh, ww, x["table"].detach() + e * to["table"], bucket, 0.5)[0]["out"] * go).sum()   # noqa: E731
    slope = (at(1e-5) - at(-1e-5)) / 2e-5
    mine = sum((val[m] * to[n]).sum() for n, m in (("q", "g_q"), ("k", "g_k"), ("v", "g_v"), ("table", "g_table")))
    assert abs(slope - mine) <= 1e-7 * sum((val[m] * to[n]).abs().sum() for n, m in (("q", "g_q"), ("k", "g_k"), ("v", "g_v"), ("table", "g_table"))) + 1e-9


def test_rows_without_keys_in_the_formulas():
    x = torch.randn(1, 1, 6, 4, dtype=torch.float64)
    table = torch.full((11, 1), -math.inf, dtype=torch.float64)
    val, _ = ref.attention(x, x, x, 1, 1, 6, table, None, 1.0, x)
    assert all((val[n] == 0).all() for n in ("out", "g_q", "g_k", "g_v", "g_table")) and (val["lse"] == -math.inf).all()


Q, K, V, O, T, BK, LSE, WS = (0x10000000 * i for i in range(1, 9))   # never dereferenced
NULL, SHAPE, UNSUPPORTED, ALIGN, ALIAS, WORKSPACE = 1, 2, 3, 4, 5, 6


def test_attention_refusals(L):
    def fwd(q=Q, k=K, v=V, B=1, heads=4, d=16, H=32, W=32, step=192, wh=16, ww=16, t=T, bk=None, n=961, scale=0.25, out=O, lse=LSE, dt=1):
        return L.esc_window_attention_forward(q, k, v, B, heads, d, H, W, step, wh, ww, t, bk, n, scale, out, lse, dt, None)

    assert fwd(q=None) == fwd(k=None) == fwd(v=None) == fwd(out=None) == NULL
    assert fwd(B=0) == fwd(heads=0) == fwd(d=0) == fwd(H=-1) == fwd(W=0) == fwd(wh=0) == fwd(ww=-2) == SHAPE
    assert fwd(step=63) == fwd(n=960) == fwd(n=0, bk=BK) == SHAPE
    assert fwd(d=65) == fwd(wh=65, ww=65, n=129 * 129) == fwd(wh=2 ** 30, bk=BK) == fwd(dt=2) == fwd(heads=70000, step=70000 * 16) == UNSUPPORTED
    assert fwd(scale=0.0) == fwd(scale=-1.0) == fwd(scale=math.nan) == fwd(scale=math.inf) == fwd(scale=1e-7) == UNSUPPORTED
    assert fwd(q=Q + 1) == fwd(t=T + 1) == fwd(out=O + 8) == fwd(lse=LSE + 2) == fwd(bk=BK + 2, n=9) == ALIGN
    assert fwd(out=Q) == fwd(out=K + 192 * 2 * 1023 + 112) == fwd(lse=O) == fwd(lse=V + 64) == ALIAS
    assert fwd(B=2 ** 30, H=2 ** 20, W=2 ** 20) == SHAPE
    assert fwd(B=2 ** 31 - 1, H=1, W=1, wh=1, ww=1, n=1, heads=8) in (SHAPE, UNSUPPORTED)


def test_attention_backward_refusals(L):
    GO, GQ, GT = 0x100000000, 0x110000000, 0x120000000
    big = 1 << 30

    def bwd(q=Q, out=O, lse=LSE, go=GO, gq=GQ, gk=GQ + 128, gv=GQ + 256, gt=GT, t=T, ws=WS, wsb=big, d=16, step=192, dt=1, H=32):
        return L.esc_window_attention_backward(q, K, V, 1, 4, d, H, 32, step, 16, 16, t, None, 961, 0.25, out, lse, go, gq, gk, gv, gt, dt, ws, wsb, None)

    assert bwd(out=None) == bwd(lse=None) == bwd(go=None) == bwd(gq=None) == bwd(gk=None) == bwd(gv=None) == bwd(t=None) == NULL
    assert bwd(d=66, step=400) == bwd(dt=5) == UNSUPPORTED
    assert bwd(step=10) == bwd(H=0) == SHAPE
    assert bwd(go=GO + 8) == bwd(out=O + 2) == bwd(gq=GQ + 1) == bwd(gt=GT + 1) == ALIGN
    assert bwd(gk=GQ) == bwd(gk=GQ + 126) == bwd(gv=GQ + 384 * 5) == bwd(gq=Q) == bwd(gk=GO) == bwd(gq=O + 64) == ALIAS
    assert bwd(ws=None) == bwd(ws=WS + 64) == bwd(wsb=1000) == WORKSPACE
    size = L.esc_window_attention_backward_workspace_bytes
    assert size(1, 4, 16, 32, 32, 16, 16) >= 32 * 32 * 4 * 4 and size(1, 4, 16, 32, 32, 16, 16) % 256 == 0
    assert size(0, 4, 16, 32, 32, 16, 16) == size(1, 4, 65, 32, 32, 16, 16) == size(1, 4, 16, 32, 32, 0, 16) == size(1, 1, 16, 9, 9, 100, 100) == 0


def test_bias_refusals(L):
    def fwd(t=T, bk=None, n=961, heads=4, wh=16, ww=16, out=O, dt=0):
        return L.esc_relpos_bias_forward(t, bk, n, heads, wh, ww, out, dt, None)

    def bwd(g=O, bk=None, n=961, heads=4, wh=16, ww=16, gt=T, dt=0, ws=WS, wsb=1 << 30):
        return L.esc_relpos_bias_backward(g, bk, n, heads, wh, ww, gt, dt, ws, wsb, None)

    for f in (fwd, bwd):
        assert f(heads=0) == f(wh=0) == f(ww=-1) == f(n=960) == f(n=0, bk=BK) == SHAPE
        assert f(dt=2) == f(wh=65, ww=65, n=129 * 129) == f(ww=8193, wh=1, n=16385) == UNSUPPORTED
        assert f(t=T + 2) == ALIGN if f is fwd else f(gt=T + 2) == ALIGN
        assert f(bk=BK + 1, n=4) == ALIGN
    assert fwd(t=None) == fwd(out=None) == bwd(g=None) == bwd(gt=None) == NULL
    assert fwd(out=O + 8) == ALIGN and fwd(out=T + 16) == ALIAS and bwd(g=T + 16) == ALIAS
    assert bwd(ws=None) == bwd(ws=WS + 8) == bwd(wsb=64) == WORKSPACE
    assert L.esc_relpos_bias_workspace_bytes(4, 16, 16) > 0 and L.esc_relpos_bias_workspace_bytes(4, 100, 100) == 0


def test_adamw_refusals(L):
    def arr(*p):
        return (ctypes.c_void_p * len(p))(*p)

    sizes = (ctypes.c_longlong * 2)(1000, 5000)
    n = ctypes.c_longlong()
    assert L.esc_adamw_plan_bytes(2, sizes) == 256 * -(-(1 + 3) * 64 // 256)
    assert L.esc_adamw_plan_bytes(0, sizes) == L.esc_adamw_plan_bytes(2, None) == L.esc_adamw_plan_bytes(1, (ctypes.c_longlong * 1)(-1)) == 0
    assert L.esc_adamw_plan_bytes(1, (ctypes.c_longlong * 1)(2 ** 60)) == 0

    def init(p=(Q, K), g=(V, O), m=(T, BK), v=(LSE, WS), ms=None, vs=None, c=None, pd=0, gd=0, st=0, plan=WS, pb=1 << 20, s=sizes, cnt=n):
        return L.esc_adamw_plan_init(2, s, arr(*p), arr(*g), arr(*m), arr(*v), ms, vs, c, pd, gd, st, plan, pb, None if cnt is None else ctypes.byref(cnt), None)

    assert init(s=None) == init(cnt=None) == init(p=(Q, None)) == init(g=(None, O)) == init(m=(T, None)) == init(v=(None, WS)) == init(st=1) == NULL
    assert init(pd=2) == init(gd=7) == init(st=2) == UNSUPPORTED
    assert init(s=(ctypes.c_longlong * 2)(4, -4)) == SHAPE
    assert init(p=(Q + 2, K)) == init(g=(V, O + 1)) == init(m=(T + 2, BK)) == init(c=arr(Q + 1, K)) == ALIGN
    assert init(st=1, ms=arr(Q, K), vs=arr(Q + 2, K)) == ALIGN
    assert init(plan=None) == init(plan=WS + 8) == init(pb=100) == WORKSPACE

    def step(plan=WS, chunks=4, pd=0, gd=0, st=0, t=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.01, gs=1.0, sc=None, sk=None):
        return L.esc_adamw_step(plan, chunks, pd, gd, st, t, lr, b1, b2, eps, wd, gs, sc, sk, None)

    assert step(plan=None) == NULL and step(plan=WS + 16) == WORKSPACE and step(sc=Q + 2) == step(sk=Q + 1) == ALIGN
    assert step(chunks=-1) == step(t=0) == step(lr=-1.0) == step(lr=math.nan) == step(b1=1.0) == step(b2=-0.1) == step(eps=-1.0) == step(wd=-0.5) == SHAPE
    assert step(pd=3) == step(gd=-1) == step(st=5) == UNSUPPORTED
    assert step(chunks=0) == 0                                           # nothing to do, nothing launched
    out = (ctypes.c_float * 4)()
    assert L.esc_adamw_scalars(3, 1e-3, 0.9, 0.99, 0.1, 2.0, out) == 0 and L.esc_adamw_scalars(0, 1e-3, 0.9, 0.99, 0.1, 2.0, out) == SHAPE
    f32 = lambda x: ctypes.c_float(x).value   # noqa: E731
    assert list(out) == [f32(1 - 1e-4), f32(1e-3 / (1 - 0.9 ** 3)), f32(1 / math.sqrt(1 - 0.99 ** 3)), 2.0]
