"""Where ReLU's slope is zero nothing of grad_out passes: an infinity or a NaN there gives the bits that a zero gives, in every kernel."""
import pytest
import torch

from tests.test_gpu_linear import make, pkg   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,N", [(5, 64, 96), (300, 64, 96), (300, 61, 97), (700, 320, 640)])   # a few rows; small layers; odd ones; wide ones
def test_what_relu_stops(pkg, dtype, rows, K, N):   # noqa: F811
    s = make(rows, K, N, dtype)
    s["z"][0, :4] = torch.tensor([0.0, -0.0, 0.0, -0.0])
    stopped = s["z"] <= 0
    assert stopped.any() and not stopped.all()
    results = []
    for value in (0.0, float("inf"), float("-inf"), float("nan")):
        go = torch.where(stopped, torch.full_like(s["go"], value), s["go"])
        got = [torch.full_like(s["x"], 7.0), torch.full((N, K), 7.0, device="cuda"), torch.full((N,), 7.0, device="cuda")]
        pkg.esc_linear_backward(s["x"], s["w"], s["z"], pkg.ESC_ACT_RELU, go, *got)
        results.append(got)
    assert all(t.isfinite().all() for t in results[0])
    for got in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], got))
