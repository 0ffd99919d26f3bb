"""How far the bf16 backward pass may be off where a row's softmax has few keys or one that dominates: its ds are small beside go . out, so D
from an `out` that was rounded to bf16 would be most of the error.

Bounds per value, with u = 2^-24, h = 2^-8 and r (p's relative error) as in attention_ref, first order in h but for the last term:
  D       the rounded out only starts it; what the row's ds add up to puts it right.  Left: p and dp in fp32, (r + 2 n u)(sum p |dp| + 2 |D|)
          + (d + 2) u sum p |go||v|, and u of each of them once more for the sums
  ds      p ((r + n u)(|dp| + |D|) + (d + 2) u |go||v| + that)
  g_q     scale sum_j (ds' error + h |ds| + 2 h p E)|k| + h |g_q|, E = what D of the rounded out may be off (it scales two roundings to bf16)
  g_k     scale sum_i (ds' error + h |ds|)|q| + h |g_k|"""
import pytest
import torch

from tests.attention_ref import H8, TINY, U, bias_matrix, check
from tests.test_gpu_window_attention import inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def tight(x, shape, scale):
    """Gradients of q and k of maps that are one window each, in 64 bits, with the bounds above."""
    B, H, W, heads, d, wh, ww = shape
    n = H * W
    cut = lambda t: t.double().reshape(B, n, heads, d).transpose(1, 2)             # noqa: E731
    back = lambda t: t.transpose(1, 2).reshape(B, H, W, heads * d)                 # noqa: E731
    q, k, v, go = (cut(x[t]) for t in ("q", "k", "v", "go"))
    bias = bias_matrix(x["table"], x["bucket"], wh, ww, H, W)
    s = scale * q @ k.transpose(2, 3) + bias
    p = torch.softmax(s, 3)
    out, dp = p @ v, go @ v.transpose(2, 3)
    D = (p * dp).sum(3, keepdim=True)
    ds = p * (dp - D)
    A = (scale * q.abs() @ k.abs().transpose(2, 3) + bias.abs()).amax((2, 3), keepdim=True)
    r = 2 * U * ((d + 3) * A + 4 * s.abs().amax((2, 3), keepdim=True) + 8)
    gv = go.abs() @ v.abs().transpose(2, 3)
    mag = (p * dp.abs()).sum(3, keepdim=True) + 2 * D.abs()
    e_D = (r + (2 * n + 4) * U) * mag + (d + 2) * U * (p * gv).sum(3, keepdim=True)
    e_ds = p * ((r + n * U) * (dp.abs() + D.abs()) + (d + 2) * U * gv + e_D) + 2 * U * ds.abs() + TINY * (dp.abs() + D.abs() + 1)
    E = (go.abs() * (h_of(out) + (r + 2 * n * U + H8) * (p @ v.abs()))).sum(3, keepdim=True)
    g_q, g_k = scale * ds @ k, scale * ds.transpose(2, 3) @ q
    op = e_ds + (H8 + 2 * n * U) * ds.abs()
    far_q = scale * (op + 2 * H8 * p * E) @ k.abs() + (H8 + 2 * U) * g_q.abs() + TINY
    far_k = scale * op.transpose(2, 3) @ q.abs() + (H8 + 2 * U) * g_k.abs() + TINY
    return {"g_q": back(g_q), "g_k": back(g_k)}, {"g_q": back(far_q), "g_k": back(far_k)}


def h_of(out):
    return H8 * out.abs()


@pytest.mark.parametrize("spread", [1.0, 3.0])
@pytest.mark.parametrize("shape", [
    (2, 1, 2, 3, 32, 16, 24), (3, 2, 2, 4, 48, 8, 8), (2, 1, 6, 2, 30, 1, 6), (2, 3, 6, 4, 16, 8, 8), (1, 1, 90, 2, 10, 1, 100),
    (1, 12, 15, 2, 8, 12, 16), (2, 16, 16, 3, 16, 16, 16), (1, 17, 11, 2, 64, 17, 11), (1, 1, 300, 2, 32, 1, 333)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_rows_that_few_keys_decide(pkg, shape, spread):
    scale = shape[4] ** -0.5
    x = inputs(shape, "bf16", 50 + sum(shape), spread=spread)
    got = run(pkg, x, shape, scale)
    val, far = tight(x, shape, scale)
    for n in val:
        check(got[n], val[n], far[n], n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(2, 1, 50, 3, 16, 1, 1), (1, 1, 1, 2, 32, 8, 8), (3, 5, 9, 2, 24, 4, 8), (1, 7, 7, 2, 64, 3, 6)], ids=lambda s: "x".join(map(str, s)))
def test_windows_of_one_pixel_have_no_gradient_of_scores(pkg, shape, dtype):
    """p is 1 whatever the score is: zeros, not the difference of two roundings of one number.  Whole windows of one pixel, a map of one, and the
    corner that the border leaves of a larger window."""
    B, H, W, heads, d, wh, ww = shape
    x = inputs(shape, dtype, 60)
    got = run(pkg, x, shape, 0.25)
    corner = {n: got[n][:, H - 1:, W - 1:] for n in ("g_q", "g_k")}          # the last pixel is a window of its own in all of these
    assert all((t == 0).all() for t in corner.values())
    if wh * ww == 1 or H * W == 1:
        assert all((got[n] == 0).all() for n in ("g_q", "g_k", "g_table"))
