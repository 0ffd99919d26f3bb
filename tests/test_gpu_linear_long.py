"""Linear layers of bf16 results over long contractions, whose terms all have one sign: what the tensor cores cut off must not add up to more than the
results' own rounding.  Bounds: tests/layers_close.py."""
import pytest
import torch

from tests import layers_close as close
from tests import layers_ref as ref
from tests.test_gpu_linear import backward, forward, make, pkg   # noqa: F401
from tests.test_gpu_linear_close import positive

pytestmark = pytest.mark.gpu


def drift(got, want):
    """Mean and largest of the relative errors: what sums of one sign lose, as far as the mean of the results' own roundings (2^-8 at most, 2^-9.8 in the
    mean of squares) does not hide it; rows and columns are of different sizes, so that these come out even."""
    off = (got.double() - want) / want
    return abs(off.mean().item()) - 5 * 2.0 ** -9.8 / (got.numel() / 4) ** 0.5, off.abs().max().item()


def sizes(n, octaves):
    return 2 ** torch.linspace(0, octaves, n, device="cuda")


@pytest.mark.parametrize("terms", [32768, 65536 + 128, 1 << 18])
def test_long_bf16_results_of_one_sign(pkg, terms):   # noqa: F811
    """Forward, and the gradient of x: a contraction of so many terms.  """
    a, b = 300, 512
    x, w = positive(4, (a, terms), (b, terms))
    x, w = (x * sizes(a, 1.7)[:, None]).bfloat16(), (w * sizes(b, 3)[:, None]).bfloat16()
    want = x.double() @ w.double().t()
    for back in (False, True):
        out = torch.empty(a, b, dtype=torch.bfloat16, device="cuda")
        if back:
            pkg.esc_linear_backward(torch.zeros_like(out), w.t().contiguous(), None, 0, x, out)
        else:
            pkg.esc_linear_forward(x, w, None, 0, out)
        mean, most = drift(out, want)
        assert mean <= close.long_run(terms) and most <= close.H8 + 2 * close.long_run(terms), back


@pytest.mark.parametrize("rows,K,N", [(1 << 17, 1536, 1536), (148 * 128 * 1024, 64, 64)])   # three kernels, with as many tiles as SMs; one pass
def test_long_bf16_gradients_of_one_sign(pkg, rows, K, N):   # noqa: F811
    """bf16 gradients of the weights over many rows."""
    go, x = positive(5, (rows, N), (rows, K))
    go, x = (go * sizes(N, 17.1)).bfloat16(), (x * sizes(K, 3)).bfloat16()
    gw, gx = torch.empty(N, K, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    pkg.esc_linear_backward(x, torch.zeros_like(gw), None, 0, go, gx, gw)
    some = min(N, 64)                                                     # outputs, for the sums in 64 bits
    want = sum(go[r:r + (1 << 20), :some].double().t() @ x[r:r + (1 << 20)].double() for r in range(0, rows, 1 << 20))
    mean, most = drift(gw[:some], want)
    assert mean <= close.long_run(32768) + 40 * close.U and most <= close.H8 + 2 * close.long_run(32768)   # 40: parts, added


@pytest.mark.parametrize("rows,K,N,pad", [(130, 33000, 136, 0), (20, 32776, 40, 8), (131, 33001, 67, 0), (300, 40000, 61, 0), (50, 65544, 72, 3)])
def test_long_bf16_sums_beside_the_epilogue(pkg, rows, K, N, pad):   # noqa: F811
    """Rows of whole pieces and others, with bias, residual, activation and z, both ways."""
    s = make(rows, K, N, "bf16", pad)
    for act in ("none", "gelu"):
        forward(pkg, s, act)
    forward(pkg, s, "relu", False, True, False)
    t = make(rows, N, K, "bf16")                                          # the gradient of x sums over so many outputs
    backward(pkg, t, "gelu")
    backward(pkg, t, "none", torch.float32)


@pytest.mark.parametrize("rows,K,N,act", [(40000, 1536, 1536, 0), (200000, 320, 72, 2), (148 * 128 * 260, 64, 64, 0)])
def test_nothing_behind_the_workspace(pkg, rows, K, N, act):   # noqa: F811
    """bf16 gradients over so many rows that they are cut into runs; the same bits with scratch of the call's own."""
    x, w, go, z = (torch.randn(*s, device="cuda").bfloat16() for s in ((rows, K), (N, K), (rows, N), (rows, N)))
    n = pkg.esc_linear_backward_workspace_bytes(rows, K, N, act, torch.bfloat16)
    ws = torch.full((n + 4096,), 123, dtype=torch.uint8, device="cuda")
    results = []
    for scratch in (ws[:n], None):
        got = [torch.empty_like(x), torch.empty_like(w), torch.empty(N, dtype=torch.bfloat16, device="cuda")]
        pkg.esc_linear_backward(x, w, z if act else None, act, go, *got, scratch)
        results.append(got)
    assert (ws[n:] == 123).all()
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert close.rel(results[0][1], ref.linear_grad(x, w, z, ["none", "relu", "gelu"][act], go, True)[0]["gw"]) <= 2 * close.H8
