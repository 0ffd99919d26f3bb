"""Linear layers and the norm's gradients as wholes, in norm, against the formulas in 64 bits: bounds so close (tests/layers_close.py) that a product of
parts, a run of a sum or a tile of rows that is missing shows (tests/test_close_cpu.py)."""
import pytest
import torch

from tests import layers_close as close
from tests import layers_ref as ref
from tests.close_cases import FP32_SIZES, GRAD_H, GRAD_SUMS, LONG, MANY_ROWS, NORM_ROWS, SMALL_ROWS, SMALL_SIZES
from tests.test_gpu_linear import pkg   # noqa: F401

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def signs(seed, *shapes):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*s, generator=g, device="cuda") for s in shapes]


def positive(seed, *shapes):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.rand(*s, generator=g, device="cuda") + 0.5 for s in shapes]


@pytest.mark.parametrize("rows,K,N", FP32_SIZES)
def test_fp32_products(pkg, rows, K, N):   # noqa: F811
    x, w, go = signs(rows, (rows, K), (N, K), (rows, N))
    out, gx, gw = torch.empty_like(go), torch.empty_like(x), torch.empty_like(w)
    pkg.esc_linear_forward(x, w, None, 0, out)
    pkg.esc_linear_backward(x, w, None, 0, go, gx, gw)
    xd, wd, gd = x.double(), w.double(), go.double()
    assert close.rel(out, xd @ wd.t()) <= close.random_signs(K)
    assert close.rel(gx, gd @ wd) <= close.random_signs(N)
    assert close.rel(gw, gd.t() @ xd) <= close.random_signs(rows, -(-rows // 64))


@pytest.mark.parametrize("a,terms,b,_", LONG)
def test_long_fp32_sums_of_one_sign(pkg, a, terms, b, _):   # noqa: F811
    """Each product with its long side as contraction; the others a and b."""
    x, w = positive(a, (a, terms), (b, terms))
    out = torch.empty(a, b, device="cuda")
    pkg.esc_linear_forward(x, w, None, 0, out)
    assert close.rel(out, x.double() @ w.double().t()) <= close.one_sign(terms)
    go, w = x, w.t().contiguous()                                         # [a, N], [N, b]
    gx = torch.empty(a, b, device="cuda")
    pkg.esc_linear_backward(torch.empty(a, b, device="cuda"), w, None, 0, go, gx)
    assert close.rel(gx, go.double() @ w.double()) <= close.one_sign(terms)
    go, x = go.t().contiguous(), w                                        # [rows, a], [rows, b]
    gw = torch.empty(a, b, device="cuda")
    pkg.esc_linear_backward(x, torch.empty(a, b, device="cuda"), None, 0, go, None, gw)
    assert close.rel(gw, go.double().t() @ x.double()) <= close.one_sign(terms, 64)


def test_long_bf16_gradient_of_one_sign(pkg):   # noqa: F811
    """144 tiles: a sum over all rows each, and its runs."""
    rows, K, N = 32768, 1536, 1536
    x, w, go = (t.bfloat16() for t in positive(3, (rows, K), (N, K), (rows, N)))
    gw = torch.empty(N, K, device="cuda")
    pkg.esc_linear_backward(x, w, None, 0, go, None, gw)
    assert close.rel(gw, go.double().t() @ x.double()) <= close.one_sign(rows, 64)


def gradients(pkg, rows, K, N, dtype, act):   # noqa: F811
    x, w, go, z = (t.to(DTYPES[dtype]) for t in signs(rows + K, (rows, K), (N, K), (rows, N), (rows, N)))
    gx, gw, gb = torch.empty_like(x), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    pkg.esc_linear_backward(x, w, z if act else None, act, go, gx, gw, gb)
    g, _ = ref.linear_grad(x, w, z, ["none", "relu", "gelu"][act], go, False)
    rounded = dtype == "bf16" and act
    assert close.rel(gw, g["gw"]) <= (GRAD_H if rounded else GRAD_SUMS), ("gw", act)
    assert close.rel(gb, g["gb"]) <= GRAD_SUMS, ("gb", act)
    assert close.rel(gx, g["gx"]) <= (2 * close.H8 if dtype == "bf16" else GRAD_SUMS), ("gx", act)


@pytest.mark.parametrize("rows", SMALL_ROWS)
@pytest.mark.parametrize("K,N", SMALL_SIZES)
def test_gradients_over_many_rows_in_one_pass(pkg, rows, K, N):   # noqa: F811
    for act in range(3):
        gradients(pkg, rows, K, N, "bf16", act)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,N", MANY_ROWS)
def test_gradients_over_many_rows(pkg, rows, K, N, dtype):   # noqa: F811
    for act in range(3):
        gradients(pkg, rows, K, N, dtype, act)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,C", NORM_ROWS)
def test_gradients_of_the_norm(pkg, rows, C, dtype):   # noqa: F811
    x, w, gy = (t.to(DTYPES[dtype]) for t in signs(rows + C, (rows, C), (C,), (rows, C)))
    gx, gw, gb = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    pkg.esc_layer_norm_backward(x, w, 1e-6, gy, gx, gw, gb)
    val, _ = ref.norm(x, w, None, 1e-6, gy)
    assert close.rel(gw, val["gw"]) <= GRAD_SUMS and close.rel(gb, val["gb"]) <= GRAD_SUMS
    assert close.rel(gx, val["gx"]) <= (2 * close.H8 if dtype == "bf16" else GRAD_SUMS)


@pytest.mark.parametrize("scale", [-104, -112, -120, -124])
@pytest.mark.parametrize("rows,K,N", [(130, 64, 96), (75, 61, 70)])
def test_small_fp32_values(pkg, rows, K, N, scale):   # noqa: F811
    """bf16 has no bits below 2^-133: a value as three parts is off by 2^-134 at most, whatever its size."""
    x, w, go = signs(rows, (rows, K), (N, K), (rows, N))
    small, large = 2.0 ** scale, 2.0 ** 100
    out, gx, gw = torch.empty_like(go), torch.empty_like(x), torch.empty_like(w)
    pkg.esc_linear_forward(x * small, w * large, None, 0, out)
    pkg.esc_linear_backward(x * large, w * large, None, 0, go * small, gx, gw)
    for name, got, a, b in (("out", out, x * small, (w * large).t()), ("gx", gx, go * small, w * large), ("gw", gw, (go * small).t(), x * large)):
        a, b = a.double(), b.double()
        bound = 2.0 ** -134 * b.abs().sum(0) + 2 * (a.shape[1] + 2) * close.U * (a.abs() @ b.abs())
        worst = ((got.double() - a @ b).abs() / bound).max().item()
        assert worst <= 1, (name, worst)
