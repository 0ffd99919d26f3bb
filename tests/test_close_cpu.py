"""The bounds of tests/layers_close.py: what the kernels do lies within them, what a mistake would make of it does not."""
import pytest
import torch

from tests import layers_close as close
from tests.close_cases import FP32_SIZES, GRAD_H, GRAD_SUMS, LONG, MANY_ROWS, NORM_ROWS, SMALL_ROWS


@pytest.mark.parametrize("rows,K,N", FP32_SIZES)
def test_every_product_of_parts_counts(rows, K, N):
    """Forward and both gradients: six products are within the bound (of their sums' own errors nothing is used up here), any five are not."""
    g = torch.Generator().manual_seed(rows)
    x, w, go = torch.randn(rows, K, generator=g), torch.randn(N, K, generator=g), torch.randn(rows, N, generator=g)
    for a, b in ((x, w), (go, w.t()), (go.t(), x.t())):
        terms = a.shape[1]
        want = a.double() @ b.double().t()
        bound = close.random_signs(terms)
        assert close.rel(close.product(a, b, close.SIX), want) <= 2 * close.U
        for left in close.SIX[3:]:
            assert close.rel(close.product(a, b, [p for p in close.SIX if p != left]), want) > 1.2 * bound, (left, terms)


@pytest.mark.parametrize("terms", sorted({t for *_, t in LONG}))
def test_sums_that_do_not_end_drift(terms):
    """Cut off with every 16 terms, to the end: even half of what that loses (the tensor cores lose less than a cut) is beyond the bound."""
    g = torch.Generator().manual_seed(terms)
    v = (torch.rand(64, terms, generator=g) + 0.5).double() * (torch.rand(64, terms, generator=g) + 0.5).double()
    want = v.sum(-1)
    assert close.rel(close.truncated(v, close.RUN), want) <= close.one_sign(terms)
    assert close.rel(close.truncated(v, terms), want) / 2 > close.one_sign(terms)


@pytest.mark.parametrize("rows", sorted({r for r, *_ in MANY_ROWS} | set(SMALL_ROWS) | {r for r, _ in NORM_ROWS}))
def test_what_is_left_out_is_seen(rows):
    """A gradient of zeros, one of the other sign, one of which 128 rows are missing, or count twice: all beyond the widest bound of the gradients."""
    g = torch.Generator().manual_seed(rows)
    go, x = torch.randn(rows, 12, generator=g).double(), torch.randn(rows, 12, generator=g).double()
    bound = max(GRAD_SUMS, GRAD_H)
    for rows_of in (lambda r: go[r].t() @ x[r], lambda r: go[r].sum(0)):
        want = rows_of(slice(0, rows))
        for first in (0, rows // 2 // 128 * 128, (rows - 1) // 128 * 128):
            lost = rows_of(slice(first, min(first + 128, rows)))
            # a last tile of a few rows is as little as it is: held to the part of it that its rows are
            few = min(1.0, (rows - first) / 128) ** 0.5
            assert (lost.norm() / want.norm()).item() > 1.2 * bound * few, (rows, first)
        assert close.rel(torch.zeros_like(want), want) > bound and close.rel(-want, want) > bound
