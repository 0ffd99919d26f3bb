"""The formulas that the GPU tests hold the layer norm and the linear layers to, against automatic differentiation and differences, and what
the entry points refuse on the host, before anything could be launched."""
import pytest
import torch

from tests import layers_ref as ref


@pytest.fixture(scope="module")
def L():
    from paper_2503_06671_b200 import build, lib

    build.build()
    return lib()


@pytest.mark.parametrize("rows,C", [(1, 1), (3, 2), (5, 7), (2, 33)])
def test_norm_formulas(rows, C):
    g = torch.Generator().manual_seed(rows * C)
    rand = lambda *n: torch.randn(*n, generator=g, dtype=torch.float64)   # noqa: E731
    x, w, b = (t.requires_grad_() for t in (rand(rows, C), rand(C), rand(C)))
    gy, skip, eps = rand(rows, C), rand(rows, C), 0.1
    y = torch.nn.functional.layer_norm(x, (C,), w, b, eps)
    gx, gw, gb = torch.autograd.grad((y * gy).sum() + (x * skip).sum(), (x, w, b))
    val, far = ref.norm(x.detach(), w.detach(), b.detach(), eps)
    assert torch.allclose(val["y"], y.detach(), rtol=0, atol=1e-12) and (far["y"] >= 0).all()
    val, far = ref.norm(x.detach(), w.detach(), None, eps, gy, skip)
    for n, t in (("gx", gx), ("gw", gw), ("gb", gb)):
        assert torch.allclose(val[n], t, rtol=0, atol=1e-12) and (far[n] >= 0).all(), n
    to, at = rand(rows, C), lambda e: ((ref.norm(x.detach() + e * to, w.detach(), b.detach(), eps)[0]["y"] * gy).sum() + ((x.detach() + e * to) * skip).sum())   # noqa: E731
    assert abs((at(1e-5) - at(-1e-5)) / 2e-5 - (val["gx"] * to).sum()) <= 1e-7 * ((val["gx"] * to).abs().sum() + 1)


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (4, 3, 5), (7, 9, 2)])
def test_linear_formulas(act, rows, K, N):
    g = torch.Generator().manual_seed(rows + K)
    rand = lambda *n: torch.randn(*n, generator=g, dtype=torch.float64)   # noqa: E731
    x, w, b, res, go = rand(rows, K).requires_grad_(), rand(N, K).requires_grad_(), rand(N).requires_grad_(), rand(rows, N), rand(rows, N)
    z = x @ w.t() + b
    out = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu}[act](z) + res
    grads = torch.autograd.grad((out * go).sum(), (x, w, b))
    val, far = ref.linear(x.detach(), w.detach(), b.detach(), act, res)
    assert torch.allclose(val["out"], out.detach(), rtol=0, atol=1e-12) and torch.allclose(val["z"], z.detach(), rtol=0, atol=1e-12)
    got, far = ref.linear_grad(x.detach(), w.detach(), z.detach(), act, go, False)
    for n, t in zip(("gx", "gw", "gb"), grads):
        assert torch.allclose(got[n], t, rtol=0, atol=1e-12) and (far[n] >= 0).all(), n
    to = rand(rows, K)
    at = lambda e: (ref.linear(x.detach() + e * to, w.detach(), b.detach(), act, res)[0]["out"] * go).sum()   # noqa: E731
    assert abs((at(1e-6) - at(-1e-6)) / 2e-6 - (got["gx"] * to).sum()) <= 1e-6 * ((got["gx"] * to).abs().sum() + 1)


X, W, B, Y, GY, GX, GW, GB, WS = (0x10000000 * (i + 1) for i in range(9))


def test_norm_refusals(L):
    """Fake, never dereferenced addresses: every call must fail on the host checks."""
    def fwd(x=X, xs=64, w=W, b=B, eps=1e-6, y=Y, ys=64, rows=100, C=64, dt=1):
        return L.esc_layer_norm_forward(x, xs, w, b, eps, y, ys, rows, C, dt, None)

    assert fwd(x=None) == 1 and fwd(y=None) == 1
    assert fwd(C=0) == 2 and fwd(rows=-1) == 2 and fwd(xs=63) == 2 and fwd(ys=63) == 2 and fwd(rows=1 << 60) == 2
    assert fwd(dt=2) == 3 and fwd(eps=-1.0) == 3 and fwd(eps=float("nan")) == 3 and fwd(eps=float("inf")) == 3
    assert fwd(C=(1 << 20) + 1, xs=1 << 21, ys=1 << 21) == 3
    assert fwd(x=X + 1) == 4 and fwd(w=W + 1) == 4 and fwd(b=B + 1) == 4 and fwd(y=Y + 1) == 4 and fwd(x=X + 2, dt=0) == 4
    assert fwd(y=X) == 5 and fwd(y=X + 64 * 2 * 99) == 5 and fwd(y=W) == 5 and fwd(y=B + 126) == 5
    assert fwd(y=X + 64, xs=128, ys=128) == 5 and fwd(x=X + 130, y=X, xs=128, ys=128, C=66) == 5
    assert fwd(rows=0) == 0 and fwd(rows=0, x=None, y=None) == 0

    need = L.esc_layer_norm_backward_workspace_bytes(100, 64)
    assert need > 0 and need % 256 == 0
    assert L.esc_layer_norm_backward_workspace_bytes(100, 0) == 0 and L.esc_layer_norm_backward_workspace_bytes(-1, 64) == 0

    def bwd(x=X, xs=64, w=W, eps=1e-6, gy=GY, skip=None, gx=GX, gw=GW, gb=GB, rows=100, C=64, dt=1, gdt=0, ws=WS, n=need):
        return L.esc_layer_norm_backward(x, xs, w, eps, gy, skip, gx, gw, gb, rows, C, dt, gdt, ws, n, None)

    assert bwd(x=None) == 1 and bwd(gy=None) == 1 and bwd(gx=None) == 1 and bwd(w=None) == 1
    assert bwd(C=0) == 2 and bwd(rows=-5) == 2 and bwd(xs=1) == 2
    assert bwd(dt=7) == 3 and bwd(gdt=5) == 3 and bwd(eps=-0.5) == 3
    assert bwd(gy=GY + 1) == 4 and bwd(gx=GX + 1) == 4 and bwd(skip=Y + 1) == 4 and bwd(gw=GW + 2) == 4 and bwd(gb=GB + 2) == 4
    assert bwd(gx=X) == 5 and bwd(gx=GY) == 5 and bwd(skip=GX) == 5 and bwd(gw=W) == 5 and bwd(gb=GW) == 5 and bwd(gw=GX + 64) == 5
    assert bwd(ws=None) == 6 and bwd(ws=WS + 8) == 6 and bwd(n=need - 1) == 6


def test_linear_refusals(L):
    def fwd(x=X, xs=64, w=W, b=B, act=2, res=GY, out=Y, z=GX, rows=100, K=64, N=192, dt=1):
        return L.esc_linear_forward(x, xs, w, b, act, res, out, z, rows, K, N, dt, None)

    assert fwd(x=None) == 1 and fwd(w=None) == 1 and fwd(out=None) == 1
    assert fwd(K=0) == 2 and fwd(N=0) == 2 and fwd(rows=-1) == 2 and fwd(xs=63) == 2
    assert fwd(act=3) == 3 and fwd(act=-1) == 3 and fwd(dt=2) == 3 and fwd(rows=1 << 31) == 3 and fwd(K=1 << 21, xs=1 << 21) == 3 and fwd(N=1 << 21) == 3
    assert fwd(x=X + 1) == 4 and fwd(w=W + 1) == 4 and fwd(b=B + 1) == 4 and fwd(res=GY + 1) == 4 and fwd(out=Y + 1) == 4 and fwd(z=GX + 1) == 4
    assert fwd(out=X) == 5 and fwd(out=W) == 5 and fwd(out=B) == 5 and fwd(out=GY) == 5 and fwd(z=Y) == 5 and fwd(z=X) == 5 and fwd(z=Y + 192 * 2 * 99) == 5
    assert fwd(rows=0) == 0
    assert fwd(rows=(1 << 31) - 8192, K=8, xs=8, N=1 << 20, out=1 << 50, res=None, z=None) == 3          # more tiles than a launch can count

    need = L.esc_linear_backward_workspace_bytes(100, 64, 192, 2, 1)
    assert need > 0 and need % 256 == 0
    for bad in [(-1, 64, 192, 2, 1), (100, 0, 192, 2, 1), (100, 64, -2, 2, 1), (100, 64, 192, 9, 1), (100, 64, 192, 2, 4), (1 << 31, 64, 192, 2, 1)]:
        assert L.esc_linear_backward_workspace_bytes(*bad) == 0

    def bwd(x=X, xs=64, w=W, z=Y, act=2, go=GY, gx=GX, gw=GW, gb=GB, rows=100, K=64, N=192, dt=1, gdt=0, ws=WS, n=need):
        return L.esc_linear_backward(x, xs, w, z, act, go, gx, gw, gb, rows, K, N, dt, gdt, ws, n, None)

    assert bwd(x=None) == 1 and bwd(w=None) == 1 and bwd(go=None) == 1 and bwd(z=None) == 1
    assert bwd(K=0) == 2 and bwd(N=-1) == 2 and bwd(xs=3) == 2
    assert bwd(act=4) == 3 and bwd(dt=3) == 3 and bwd(gdt=2) == 3
    assert bwd(go=GY + 1) == 4 and bwd(gx=GX + 1) == 4 and bwd(gw=GW + 2) == 4 and bwd(gb=GB + 1) == 4 and bwd(z=Y + 1) == 4
    assert bwd(gx=X) == 5 and bwd(gx=GY) == 5 and bwd(gx=W) == 5 and bwd(gx=Y) == 5 and bwd(gw=W) == 5 and bwd(gb=GW) == 5 and bwd(gw=GX) == 5
    assert bwd(ws=None) == 6 and bwd(ws=WS + 1) == 6 and bwd(n=need - 1) == 6


def test_binding_refusals(L):
    """Shapes, types and strides that the C entry could not see."""
    import paper_2503_06671_b200 as esc
    from paper_2503_06671_b200 import binding

    x, w = torch.zeros(4, 6, 8), torch.zeros(8)
    rows = lambda t: binding._rows_of("x", t)   # noqa: E731
    assert rows(x) == (24, 8, 8) and rows(x[:, :, :5]) == (24, 5, 8) and rows(x[1:3, 2:3, :4]) == (2, 4, 48) and rows(x[0, 0]) == (1, 8, 8)
    assert rows(x[:0]) == (0, 8, 8) and rows(x[:, :, :1])[:2] == (24, 1)
    for t in (x.transpose(1, 2), x[:, :3], x.expand(2, 4, 6, 8), x[:, :, ::2], torch.zeros(1, 8).expand(5, 8), x.flip(0)[..., :0]):
        with pytest.raises(ValueError):
            rows(t)
    for call in (lambda: esc.esc_layer_norm_forward(x, w, w, 1e-6, x[:2]),
                 lambda: esc.esc_layer_norm_forward(x, w[:4], w, 1e-6, torch.zeros_like(x)),
                 lambda: esc.esc_layer_norm_forward(x, w, w.double(), 1e-6, torch.zeros_like(x)),
                 lambda: esc.esc_layer_norm_forward(x, w, w, 1e-6, torch.zeros_like(x)),                   # not on a GPU
                 lambda: esc.esc_layer_norm_backward(x, w, 1e-6, x[:, :, :4], torch.zeros_like(x)),
                 lambda: esc.esc_layer_norm_backward(x, w, 1e-6, x, torch.zeros_like(x), w, w[:2]),
                 lambda: esc.esc_linear_forward(x, torch.zeros(5, 7), None, 0, torch.zeros(4, 6, 5)),
                 lambda: esc.esc_linear_forward(x, torch.zeros(5, 8), torch.zeros(4), 0, torch.zeros(4, 6, 5)),
                 lambda: esc.esc_linear_forward(x, torch.zeros(5, 8), None, 0, torch.zeros(4, 6, 5).bfloat16()),
                 lambda: esc.esc_linear_backward(x, torch.zeros(5, 8), None, 0, torch.zeros(4, 6, 4)),
                 lambda: esc.esc_linear_backward(x, torch.zeros(5, 8), None, 0, torch.zeros(4, 6, 5), None, torch.zeros(8, 5)),
                 lambda: esc.new_linear_workspace(-1, 8, 8, 0, torch.float32), lambda: esc.new_layer_norm_workspace(4, 0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        esc.new_linear_workspace(4, 8, 8, 0, torch.float16)
    with pytest.raises(ValueError):
        binding._grad_code(torch.zeros(1), torch.zeros(1).bfloat16())
