"""Linear layers whose rows start anywhere and lie between values that are not numbers, against their formulas in 64 bits."""
import pytest
import torch

from tests.test_gpu_linear import backward, forward, make, pkg   # noqa: F401

pytestmark = pytest.mark.gpu


def among_nans(t, shift, pad=0):
    """The same values `shift` behind a 16-byte border, rows `pad` values further apart, NaN all around."""
    rows, width = t.shape if t.dim() == 2 else (1, t.numel())
    flat = torch.full((shift + rows * (width + pad) + 16,), float("nan"), dtype=t.dtype, device="cuda")
    new = flat[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    new.copy_(t.view(rows, width))
    return new if t.dim() == 2 else new.view(-1)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shift", range(8))
@pytest.mark.parametrize("rows,K,N,pad", [(20, 1, 3, 0), (40, 7, 9, 2), (130, 9, 63, 1), (33, 61, 65, 3), (200, 64, 64, 5), (150, 65, 129, 0), (70, 250, 777, 6), (300, 131, 8, 7)])
def test_rows_anywhere(pkg, dtype, shift, rows, K, N, pad):   # noqa: F811
    s = make(rows, K, N, dtype)
    s = {k: among_nans(t, shift, pad if k == "x" else 0) for k, t in s.items()}
    forward(pkg, s, "gelu")
    backward(pkg, s, "relu")
    backward(pkg, s, "none", torch.float32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("which", ["x", "w", "go", "z", "residual", "b"])
def test_one_tensor_is_not_aligned(pkg, dtype, which):   # noqa: F811
    s = make(400, 72, 136, dtype)
    s[which] = among_nans(s[which], 3)
    forward(pkg, s, "relu")
    backward(pkg, s, "gelu")


@pytest.mark.parametrize("rows,K,N", [(700, 2050, 96), (300, 1024, 260), (5000, 130, 140), (20000, 64, 200), (129, 4100, 33)])
def test_long_sums(pkg, rows, K, N):   # noqa: F811
    """fp32 sums of more than 512 values, in each of the three products, in tiles of one and several units and with a residual between them."""
    s = make(rows, K, N, "fp32")
    for residual in (False, True):
        forward(pkg, s, "none", residual=residual, keep=residual)
    backward(pkg, s, "gelu")
    s = make(rows, N, K, "fp32")
    forward(pkg, s, "relu", keep=False)
    backward(pkg, s, "none")


@pytest.mark.parametrize("rows,K,N", [(20000, 61, 64), (20000, 61, 128), (20000, 61, 129), (1100, 1001, 1100)])
def test_with_and_without_a_copy(pkg, rows, K, N):   # noqa: F811
    """Ragged bf16 rows that the backward pass takes as they are, and copies."""
    s = make(rows, K, N, "bf16", 3)
    backward(pkg, s, "gelu")
    backward(pkg, s, "none", torch.float32)
