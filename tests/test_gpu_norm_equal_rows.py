"""Layer norm of rows of equal values, and of rows far from zero: a mean that is off by a step of its own is large beside differences that are none.

Rows of one value: all differences from one of the row's values are 0, their mean is 0, y is the bias (rounded), and the weights' gradients
get nothing from such a row.
Rows far from zero: differences from one of the values, x0, are exact, and from there on their size counts, not x's.  The bounds of the row
x - base hold, twice: x0 lies 18 steps from base at most and the others 9.5 on average, so mean|x - x0| is 22 steps at most for five values (x0's own
is 0) and 28 for many; a sum of five values rounds four times, its mean once more and the difference once, 6 u 22 steps against 2 (5 + 2) u 9.5, and
for more values the sums' depth (at most n / 256 + 13 threads and shuffles) falls behind n + 2.
"""
import pytest
import torch

from tests import layers_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
# every kernel: rows of 16-byte pieces and of single values, a warp's and a block's, in registers and not
WIDTHS = [5, 20, 48, 61, 96, 112, 192, 250, 511, 777, 1032, 2047, 2056, 5001, 8200, 20001]
VALUES = [255.0, 1000.0, 3000.0, 10000.0, -333.0, 0.1, 1e-20, 7e8]


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def weights(C, dtype, seed):
    g = torch.Generator().manual_seed(seed + C)
    rand = lambda *n: torch.randn(*n, generator=g).to(DTYPES[dtype]).cuda()   # noqa: E731
    return rand(C), rand(C), rand


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_rows_of_one_value(pkg, dtype, C):
    w, b, rand = weights(C, dtype, 1)
    x = torch.tensor(VALUES)[:, None].expand(-1, C).to(DTYPES[dtype]).cuda().contiguous()
    y = torch.empty_like(x)
    pkg.esc_layer_norm_forward(x, w, b, 1e-6, y)
    assert torch.equal(y, b.expand_as(y))
    pkg.esc_layer_norm_forward(x, None, None, 1e-6, y)
    assert (y == 0).all()
    pkg.esc_layer_norm_forward(x, w, b, 0.0, y)
    assert y.isnan().all()                                                # 0 / 0, as the header says
    gy, skip = rand(len(VALUES), C), rand(len(VALUES), C)
    gx, gw, gb = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    pkg.esc_layer_norm_backward(x, w, 1e-2, gy, gx, gw, gb, skip)
    assert (gw == 0).all()
    val, far = ref.norm(torch.zeros_like(x), w, None, 1e-2, gy, skip)     # the same gradients as of rows of zeros
    for name, t in (("gx", gx), ("gb", gb)):
        ref.check(name, t, val, far)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_rows_far_from_zero(pkg, dtype, C):
    """Values of a few neighbouring steps around a large one."""
    w, b, rand = weights(C, dtype, 2)
    g = torch.Generator().manual_seed(C)
    step = torch.finfo(DTYPES[dtype]).eps                                 # from one value to the next, in [1, 2)
    base = torch.tensor([1.25, 1.5, 1.75, 1.875])[:, None] * 2.0 ** torch.tensor([0, 7, 12, 20])[:, None]
    x = (base * (1 + 2 * step * torch.randint(-9, 10, (4, C), generator=g))).to(DTYPES[dtype]).cuda()
    x[:, 0] = base[:, 0].to(x.dtype) * (1 - 16 * step)                     # never of one value
    gy, skip, eps = rand(4, C), rand(4, C), 1e-6
    y, gx, gw, gb = torch.empty_like(x), torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    pkg.esc_layer_norm_forward(x, w, b, eps, y)
    pkg.esc_layer_norm_backward(x, w, eps, gy, gx, gw, gb, skip)
    # x less a value of its own type near its mean is exact, and has the same norm: the bounds of that row hold for this one
    near = (x.double() - base.cuda().double()).float()
    assert torch.equal(near.double() + base.cuda().double(), x.double())
    for val, far, got in ((*ref.norm(near, w, b, eps), {"y": y}), (*ref.norm(near, w, None, eps, gy, skip), {"gx": gx, "gw": gw, "gb": gb})):
        for name, t in got.items():
            ref.check(name, t, val, {name: 2 * far[name]})


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_first_values_unlike_the_others(pkg, dtype, C):
    """The first value, or another one, is far from the rest, tiny beside it, or not finite: that row has the bounds of its own size, or is NaN, and
    its neighbours know nothing of it."""
    w, b, rand = weights(C, dtype, 3)
    x, gy, skip = rand(40, C), rand(40, C), rand(40, C)
    x[3] += 100
    x[3, 0], x[4, 0], x[5, 0], x[6, 0], x[7, C // 2], x[8, C - 1] = 0.0, 1e4, -3e9, 1e-30, 3e9, -1e4
    for bad in (None, float("inf"), float("-inf"), float("nan")):
        rows = list(range(40))
        if bad is not None:
            x[9, 0] = bad
            rows.remove(9)
        y, gx = torch.empty_like(x), torch.empty_like(x)
        pkg.esc_layer_norm_forward(x, w, b, 1e-5, y)
        pkg.esc_layer_norm_backward(x, w, 1e-5, gy, gx, None, None, skip)
        assert bad is None or (y[9].isnan().all() and gx[9].isnan().all())
        val, far = ref.norm(x[rows], w, b, 1e-5)
        ref.check("y", y[rows], val, far)
        val, far = ref.norm(x[rows], w, None, 1e-5, gy[rows], skip[rows])
        ref.check("gx", gx[rows], val, far)
