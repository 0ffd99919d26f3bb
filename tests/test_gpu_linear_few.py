"""Linear layers of a few rows, on both sides of where they change to the kernels of many rows, against their formulas in 64 bits."""
import pytest
import torch

from tests import layers_ref as ref
from tests.test_gpu_linear import backward, forward, make, pkg   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 8, 9, 15, 16, 17])
@pytest.mark.parametrize("K,N", [(1, 1), (3, 700), (64, 8), (33, 2500), (129, 591), (1000, 592), (2052, 17)])
def test_rows(pkg, dtype, rows, K, N):   # noqa: F811
    s = make(rows, K, N, dtype)
    forward(pkg, s, "gelu")
    forward(pkg, s, "relu", bias=False, residual=False, keep=False)
    backward(pkg, s, "gelu")
    backward(pkg, s, "none", torch.float32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,N", [(4, 4096, 2048), (5, 4096, 2048), (8, 4001, 4001), (9, 4001, 4001), (1, 10, 100000), (1, 100000, 10)])
def test_large_weights(pkg, dtype, rows, K, N):   # noqa: F811
    s = make(rows, K, N, dtype)
    forward(pkg, s, "none")
    backward(pkg, s, "relu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(1, 0), (4, 0), (8, 0), (0, 1), (0, 4)])
def test_strides_and_alignments(pkg, dtype, pad, shift):   # noqa: F811
    """Rows of x inside a wider tensor; every tensor behind a 16-byte border."""
    s = make(7, 72, 50, dtype, pad)
    if shift:
        for k, t in s.items():
            flat = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
            s[k] = flat[shift:].view(t.shape).copy_(t)
    for want in (("gx", "gw", "gb"), ("gx",), ("gw",), ("gb",)):
        backward(pkg, s, "gelu", torch.float32, want)
    forward(pkg, s, "gelu")


def test_grad_weight_alone_is_not_aligned(pkg):   # noqa: F811
    s = make(6, 64, 40, "bf16")
    val, far = ref.linear_grad(s["x"], s["w"], s["z"], "none", s["go"], True)
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.full((40 * 64 + 2,), 7.0, dtype=dtype, device="cuda")
        pkg.esc_linear_backward(s["x"], s["w"], None, 0, s["go"], None, flat[1:-1].view(40, 64))
        ref.check("gw", flat[1:-1].view(40, 64), val, far)
        assert flat[0] == 7 and flat[-1] == 7


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,N", [(1, 48, 1884), (16, 130, 3001), (8, 512, 512)])
def test_nothing_behind_the_workspace(pkg, dtype, rows, K, N):   # noqa: F811
    s = make(rows, K, N, dtype)
    n = pkg.esc_linear_backward_workspace_bytes(rows, K, N, 2, s["x"].dtype)
    ws = torch.full((n + 4096,), 123, dtype=torch.uint8, device="cuda")
    gx, gw, gb = (torch.empty_like(t) for t in (s["x"], s["w"], s["b"]))
    pkg.esc_linear_backward(s["x"], s["w"], s["z"], 2, s["go"], gx, gw, gb, ws[:n])
    assert (ws[n:] == 123).all()
    again = [torch.empty_like(t) for t in (gx, gw, gb)]
    pkg.esc_linear_backward(s["x"], s["w"], s["z"], 2, s["go"], *again)
    assert all(torch.equal(a, b) for a, b in zip((gx, gw, gb), again))


def test_a_row_that_is_not_finite_stays_alone(pkg):   # noqa: F811
    for dtype in ("fp32", "bf16"):
        s = make(5, 64, 96, dtype)
        clean, out = torch.empty_like(s["go"]), torch.empty_like(s["go"])
        pkg.esc_linear_forward(s["x"], s["w"], s["b"], 2, clean)
        s["x"][4, 3] = float("nan")
        pkg.esc_linear_forward(s["x"], s["w"], s["b"], 2, out)
        assert torch.equal(out[:4], clean[:4]) and torch.isnan(out[4]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_beside_an_eager_call(pkg, dtype):   # noqa: F811
    """A head of one pooled row: norm, linear and their gradients, captured and replayed with other values."""
    s = make(3, 64, 200, "fp32" if dtype == torch.float32 else "bf16")
    y, out, z = torch.empty_like(s["x"]), torch.empty_like(s["go"]), torch.empty_like(s["go"])
    ws = pkg.new_linear_workspace(3, 64, 200, 2, dtype)
    gx, gw, gb = (torch.empty_like(t) for t in (s["x"], s["w"], s["b"]))

    def step(workspace):
        pkg.esc_layer_norm_forward(s["x"], None, None, 1e-6, y)
        pkg.esc_linear_forward(y, s["w"], s["b"], 2, out, s["residual"], z)
        pkg.esc_linear_backward(y, s["w"], z, 2, s["go"], gx, gw, gb, workspace)

    step(ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ws)
    s["x"].copy_(s["x"].flip(0) * 0.5 + 1)
    step(pkg.new_linear_workspace(3, 64, 200, 2, dtype))
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, z, gx, gw, gb)]
    for t in (out, z, gx, gw, gb):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (out, z, gx, gw, gb)))
