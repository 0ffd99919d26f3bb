"""The backward pass of small bf16 layers with fp32 gradients, over rows enough for several sums of gw in every block, against the formulas in 64 bits."""
import pytest
import torch

from tests import layers_ref as ref
from tests.test_gpu_linear import backward, make, pkg   # noqa: F401

pytestmark = pytest.mark.gpu
SMS = 148


@pytest.mark.parametrize("tiles", [1, 4, 5, 8, 9, 13])
@pytest.mark.parametrize("K,N", [(64, 64), (64, 192), (128, 128), (48, 96), (192, 64), (72, 136)])
def test_fp32_gradients(pkg, tiles, K, N):   # noqa: F811
    """`tiles` of 128 rows to a block, and a few rows less: the last blocks have one tile less."""
    s = make(tiles * SMS * 128 - 1000, K, N, "bf16")
    backward(pkg, s, "gelu", torch.float32)
    backward(pkg, s, "none", torch.float32, ("gw", "gb"))


@pytest.mark.parametrize("rows", [128 * SMS * 4, 128 * SMS * 4 + 1, 128 * SMS * 5, 128 * SMS * 9 + 77])
def test_sums_do_not_drift(pkg, rows):   # noqa: F811
    """Products of one sign, which truncated sums lose alike.  A sum ends after 512 rows: 32 additions that lose a step at most (2^-18 of the value), then
    some 4 of runs and 37 of blocks that round by half a step (2^-18.6)."""
    x, w, go = torch.rand(rows, 64), torch.rand(64, 64), torch.rand(rows, 64)
    x, w, go = (t.bfloat16().cuda() for t in (x, w, go))
    gw = torch.empty(64, 64, device="cuda")
    pkg.esc_linear_backward(x, w, None, 0, go, torch.empty_like(x), gw)
    want = go.double().t() @ x.double()
    assert ((gw.double() - want).abs() / want).max().item() <= 2.0 ** -17
    again = torch.empty_like(gw)
    pkg.esc_linear_backward(x, w, None, 0, go, None, again)
    assert torch.equal(gw, again)


def test_whole_workspace(pkg):   # noqa: F811
    s = make(128 * SMS * 6, 64, 128, "bf16")
    n = pkg.esc_linear_backward_workspace_bytes(s["x"].shape[0], 64, 128, 2, torch.bfloat16)
    ws = torch.full((n + 4096,), 123, dtype=torch.uint8, device="cuda")
    gx, gw, gb = torch.empty_like(s["x"]), torch.empty(128, 64, device="cuda"), torch.empty(128, device="cuda")
    pkg.esc_linear_backward(s["x"], s["w"], s["z"], 2, s["go"], gx, gw, gb, ws[:n])
    assert (ws[n:] == 123).all()
    val, far = ref.linear_grad(s["x"], s["w"], s["z"], "gelu", s["go"], True)
    for name, t in (("gx", gx), ("gw", gw), ("gb", gb)):
        ref.check(name, t, val, far)
