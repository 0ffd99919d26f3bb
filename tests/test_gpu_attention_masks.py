"""Where a bias ends and a mask begins: an entry of -9984 or less is a mask, a larger one is a number.  The attention is held to softmax over
the matrix that esc_relpos_bias_forward writes (which knows no masks), in 64 bits, within the bounds of attention_ref."""
import math

import pytest
import torch

from tests import attention_ref as ref
from tests.test_gpu_window_attention import DTYPES, inputs, run

pytestmark = pytest.mark.gpu

SHAPE = (1, 6, 9, 2, 16, 6, 9)           # one window


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def by_matrix(pkg, x):
    """out of softmax(scale q k^T + the matrix) v in 64 bits."""
    B, H, W, heads, d, wh, ww = SHAPE
    n = H * W
    bias = pkg.esc_relpos_bias_forward(x["table"].cuda(), None, wh, ww, torch.empty(heads, n, n, dtype=x["table"].dtype, device="cuda")).cpu().double()
    q, k, v = (x[t][0].double().reshape(n, heads, d).transpose(0, 1) for t in "qkv")
    s = 0.25 * q @ k.transpose(1, 2) + bias
    return (torch.softmax(s, 2) @ v).transpose(0, 1).reshape(1, H, W, heads * d)


def bounds(x, dtype):
    val, far = ref.attention(x["q"], x["k"], x["v"], *(SHAPE[i] for i in (3, 5, 6)), x["table"], None, 0.25, x["go"], dtype == "bf16")
    return val, far


@pytest.mark.parametrize("dtype", DTYPES)
def test_entries_above_the_threshold_are_numbers(pkg, dtype):
    """All of a row down there: softmax does not see the common shift, beyond what fp32 holds at 10^4."""
    x = inputs(SHAPE, dtype, 40)
    edge = -9984.0 + 2.0 ** -10 if dtype == "fp32" else -9920.0         # the next number
    x["table"][:] = edge
    assert float(x["table"][0, 0]) == edge > -9984.0
    x["table"][::5] = edge + 64.0                                       # some keys ahead of the others by 64
    got = run(pkg, x, SHAPE, 0.25)
    val, far = bounds(x, dtype)
    for n, t in got.items():
        ref.check(t, val[n], far[n], n)
    ref.check(got["out"], by_matrix(pkg, x), far["out"], "by the matrix")
    assert torch.isfinite(got["lse"]).all() and (got["lse"] < -9000).all()


@pytest.mark.parametrize("mask", [-9984.0, -10000.0, "lowest"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_beside_others_is_softmax_of_the_matrix(pkg, dtype, mask):
    """A row that has other keys: the mask's number and -inf give the same."""
    x = inputs(SHAPE, dtype, 41)
    mask = torch.finfo(DTYPES[dtype]).min if mask == "lowest" else mask
    x["table"][::2] = mask
    x["table"][(2 * 6 - 1) * (2 * 9 - 1) // 2] = 0.5                    # a query's own place: no row is without keys
    got = run(pkg, x, SHAPE, 0.25)
    want = by_matrix(pkg, x)
    x["table"][x["table"] <= -9984] = -math.inf
    val, far = bounds(x, dtype)
    for n, t in got.items():
        ref.check(t, val[n], far[n], n)
    ref.check(got["out"], want, far["out"], "by the matrix")


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_masks_alone(pkg, dtype):
    """At the threshold itself: zeros from the attention; the matrix keeps the number, of which softmax would be a distribution."""
    x = inputs(SHAPE, dtype, 42)
    x["table"][:] = -9984.0
    got = run(pkg, x, SHAPE, 0.25)
    assert (got["lse"] == -math.inf).all() and all((got[n] == 0).all() for n in ("out", "g_q", "g_k", "g_v", "g_table"))
    assert (by_matrix(pkg, x).abs().sum(3) > 0).all()
