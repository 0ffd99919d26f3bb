"""Layer norm, forward and backward, against its formulas in 64 bits: widths that take every kernel, odd ones, slices, rows that are hard."""
import pytest
import torch

from tests import layers_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def make(rows, C, dtype, pad=0, seed=0, off=0.5):
    g = torch.Generator().manual_seed(seed + rows + C)
    rand = lambda *n: torch.randn(*n, generator=g).to(DTYPES[dtype]).cuda()   # noqa: E731
    x = (torch.randn(rows, C + pad, generator=g) * torch.exp(torch.randn(rows, 1, generator=g)) + off).to(DTYPES[dtype]).cuda()[:, :C]
    return x, rand(C), rand(C), rand(rows, C), rand(rows, C)


def both(pkg, x, w, b, gy, skip, eps=1e-6, gdt=torch.float32, want_b=True):
    rows, C = x.shape
    y, gx = torch.full((rows, C), 7.0, dtype=x.dtype, device="cuda"), torch.full((rows, C), 7.0, dtype=x.dtype, device="cuda")
    pkg.esc_layer_norm_forward(x, w, b, eps, y)
    gw = torch.full((C,), 7.0, dtype=gdt, device="cuda") if w is not None else None
    gb = torch.full((C,), 7.0, dtype=gdt, device="cuda") if want_b else None
    pkg.esc_layer_norm_backward(x, w, eps, gy, gx, gw, gb, skip)
    torch.cuda.synchronize()
    val, far = ref.norm(x, w, b, eps)
    ref.check("y", y, val, far)
    val, far = ref.norm(x, w, None, eps, gy, skip)
    for name, t in (("gx", gx), ("gw", gw), ("gb", gb)):
        if t is not None:
            ref.check(name, t, val, far)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [1, 2, 4, 7, 8, 12, 16, 24, 31, 32, 48, 60, 64, 96, 100, 128, 180, 192, 250, 255, 256, 320, 384, 504, 511, 512, 520, 768, 1024, 1026,
                               2047, 2048, 2056, 4096])
def test_widths(pkg, dtype, C):
    x, w, b, gy, skip = make(37, C, dtype)
    both(pkg, x, w, b, gy, skip)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C", [2050, 4100, 5001, 8192, 8200, 20000])
def test_rows_that_registers_do_not_hold(pkg, dtype, C):
    x, w, b, gy, skip = make(5, C, dtype, pad=3)
    both(pkg, x, w, b, gy, skip, gdt=DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,C", [(1, 64), (2, 64), (31, 48), (33, 192), (5000, 64), (20011, 48), (3001, 777)])
def test_rows(pkg, dtype, rows, C):
    x, w, b, gy, _ = make(rows, C, dtype)
    both(pkg, x, w, b, gy, None, gdt=DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pad", [1, 2, 8])
def test_slices(pkg, dtype, pad):
    """x and y as slices of wider tensors: what lies between y's rows stays."""
    x, w, b, gy, skip = make(45, 64, dtype, pad)
    both(pkg, x, w, b, gy, skip)
    wide = torch.full((45, 64 + pad), 3.0, dtype=x.dtype, device="cuda")
    pkg.esc_layer_norm_forward(x, w, b, 1e-6, wide[:, pad:])
    y = torch.empty(45, 64, dtype=x.dtype, device="cuda")
    pkg.esc_layer_norm_forward(x, w, b, 1e-6, y)
    assert (wide[:, :pad] == 3).all() and torch.equal(wide[:, pad:], y)


def test_maps_and_missing_weights(pkg):
    x, w, b, gy, _ = make(2 * 5 * 7, 32, "bf16")
    m = x.view(2, 5, 7, 32)
    y = torch.empty_like(m)
    pkg.esc_layer_norm_forward(m, w, b, 1e-6, y)
    flat = torch.empty_like(x)
    pkg.esc_layer_norm_forward(x, w, b, 1e-6, flat)
    assert torch.equal(y.view(-1, 32), flat)
    both(pkg, x, None, None, gy, None)
    both(pkg, x, w, None, gy, None, want_b=False)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_hard_rows(pkg, dtype):
    """Rows far from zero, of one value, of zeros, tiny and large ones beside one another."""
    x, w, b, gy, skip = make(12, 96, dtype)
    x[1] += 1000
    x[2] = 3.0
    x[3] = 0.0
    x[4] *= 1e-12
    x[5] *= 1e12
    x[6, 0] = 1e4
    both(pkg, x, w, b, gy, skip, eps=1e-5)
    both(pkg, torch.cat([x[:2], x[5:]]).contiguous(), w, b, torch.cat([gy[:2], gy[5:]]), None, eps=0.0)


def test_not_finite_rows_stay_among_themselves(pkg):
    x, w, b, gy, _ = make(64, 64, "bf16")
    clean, again = torch.empty_like(x), torch.empty_like(x)
    pkg.esc_layer_norm_forward(x, w, b, 1e-6, clean)
    x[5, 3], x[9, 63] = float("nan"), float("inf")
    pkg.esc_layer_norm_forward(x, w, b, 1e-6, again)
    rest = [i for i in range(64) if i not in (5, 9)]
    assert torch.equal(clean[rest], again[rest]) and again[5].isnan().all() and again[9].isnan().any()


def test_no_rows(pkg):
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    gw, gb = torch.full((64,), 5.0, device="cuda"), torch.full((64,), 5.0, device="cuda")
    pkg.esc_layer_norm_forward(x, w, None, 1e-6, torch.empty_like(x))
    pkg.esc_layer_norm_backward(x, w, 1e-6, x, torch.empty_like(x), gw, gb)
    assert (gw == 0).all() and (gb == 0).all()


def test_same_bits(pkg):
    x, w, b, gy, skip = make(9001, 64, "bf16")
    runs = []
    for _ in range(3):
        gx, gw, gb = torch.empty_like(gy), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
        pkg.esc_layer_norm_backward(x, w, 1e-6, gy, gx, gw, gb, skip)
        runs.append((gx, gw, gb))
    for r in runs[1:]:
        assert all(torch.equal(a, c) for a, c in zip(runs[0], r))
