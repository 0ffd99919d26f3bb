"""Linear layers with bias, activation and residual, forward and backward, against their formulas in 64 bits."""
import pytest
import torch

from tests import layers_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
ACTS = ["none", "relu", "gelu"]


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def make(rows, K, N, dtype, pad=0, seed=0):
    g = torch.Generator().manual_seed(seed + rows + K + N)
    rand = lambda *n: torch.randn(*n, generator=g)   # noqa: E731
    to = lambda t: t.to(DTYPES[dtype]).cuda()   # noqa: E731
    return {"x": to(rand(rows, K + pad))[:, :K], "w": to(rand(N, K) * K ** -0.5), "b": to(rand(N)), "residual": to(rand(rows, N)),
            "go": to(rand(rows, N)), "z": to(1.5 * rand(rows, N))}


def forward(pkg, s, act, bias=True, residual=True, keep=True):
    rows, N = s["go"].shape
    new = lambda: torch.full((rows, N), 7.0, dtype=s["x"].dtype, device="cuda")   # noqa: E731
    out, z = new(), new() if keep else None
    b, res = s["b"] if bias else None, s["residual"] if residual else None
    pkg.esc_linear_forward(s["x"], s["w"], b, ACTS.index(act), out, res, z)
    torch.cuda.synchronize()
    val, far = ref.linear(s["x"], s["w"], b, act, res)
    ref.check("out", out, val, far)
    if keep:
        ref.check("z", z, val, far)


def backward(pkg, s, act, gdt=None, want=("gx", "gw", "gb")):
    (rows, K), N, dtype = s["x"].shape, s["w"].shape[0], s["x"].dtype
    gdt = gdt or dtype
    new = lambda t, *n: torch.full(n, 7.0, dtype=t, device="cuda")   # noqa: E731
    got = {"gx": new(dtype, rows, K), "gw": new(gdt, N, K), "gb": new(gdt, N)}
    pkg.esc_linear_backward(s["x"], s["w"], s["z"] if act != "none" else None, ACTS.index(act), s["go"], *(got[n] if n in want else None for n in ("gx", "gw", "gb")))
    torch.cuda.synchronize()
    val, far = ref.linear_grad(s["x"], s["w"], s["z"], act, s["go"], dtype == torch.bfloat16)
    for n in got:
        if n in want:
            ref.check(n, got[n], val, far)
        else:
            assert (got[n] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (1, 64, 64), (2, 8, 16), (17, 48, 144), (64, 16, 32), (127, 64, 192), (128, 64, 64), (129, 72, 40), (300, 192, 576),
                                      (257, 63, 65), (50, 250, 777), (33, 1024, 256), (1000, 128, 128), (515, 520, 264)])
def test_sizes(pkg, dtype, act, rows, K, N):
    s = make(rows, K, N, dtype)
    forward(pkg, s, act)
    backward(pkg, s, act)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,N", [(20000, 64, 128), (40013, 48, 64), (5000, 192, 64), (3001, 320, 640), (70000, 16, 16), (9000, 100, 36)])
def test_many_rows(pkg, dtype, rows, K, N):
    s = make(rows, K, N, dtype)
    forward(pkg, s, "gelu", keep=False)
    backward(pkg, s, "gelu", torch.float32)
    backward(pkg, s, "none")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,K,N", [(1, 1024, 2048), (3, 2048, 96), (8, 4096, 100), (16, 640, 1000), (40, 2050, 511)])
def test_few_rows(pkg, dtype, rows, K, N):
    s = make(rows, K, N, dtype)
    forward(pkg, s, "gelu")
    backward(pkg, s, "relu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pad", [1, 2, 4, 8])
@pytest.mark.parametrize("rows,K,N", [(200, 64, 64), (200, 61, 67)])
def test_slices(pkg, dtype, pad, rows, K, N):
    s = make(rows, K, N, dtype, pad)
    forward(pkg, s, "relu")
    backward(pkg, s, "gelu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("keep", [False, True])
def test_epilogue(pkg, dtype, bias, residual, keep):
    s = make(150, 80, 96, dtype)
    for act in ACTS:
        forward(pkg, s, act, bias, residual, keep)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("want", [("gx",), ("gw",), ("gb",), ("gx", "gb"), ("gw", "gb")])
def test_some_gradients(pkg, dtype, want):
    s = make(300, 64, 96, dtype)
    for act in ACTS:
        backward(pkg, s, act, torch.float32, want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_unaligned_tensors(pkg, dtype):
    """Every tensor one value behind a 16-byte border."""
    s = make(140, 64, 96, dtype)
    for k, t in s.items():
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        s[k] = flat[1:].view(t.shape).copy_(t)
    forward(pkg, s, "gelu")
    backward(pkg, s, "gelu")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_far_values(pkg, dtype):
    """GELU and its slope far out on both sides; the slope of ReLU at zero is zero."""
    s = make(64, 32, 64, dtype)
    s["z"][0] = torch.linspace(-40, 40, 64)
    s["z"][1] = torch.linspace(-1e4, 1e4, 64)
    s["z"][2], s["z"][3] = 0.0, -0.0
    s["x"][5] *= 1e3
    for act in ACTS:
        forward(pkg, s, act)
        backward(pkg, s, act)


def test_not_finite_rows_stay_among_themselves(pkg):
    for dtype in DTYPES:
        s = make(300, 64, 96, dtype)
        clean, again = torch.empty_like(s["go"]), torch.empty_like(s["go"])
        pkg.esc_linear_forward(s["x"], s["w"], s["b"], 2, clean)
        s["x"][7, 3], s["x"][200, 63] = float("nan"), float("inf")
        pkg.esc_linear_forward(s["x"], s["w"], s["b"], 2, again)
        rest = [i for i in range(300) if i not in (7, 200)]
        assert torch.equal(clean[rest], again[rest]) and again[7].isnan().all() and not again[200].isfinite().all()


def test_no_rows(pkg):
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(32, 64, device="cuda")
    out, gw, gb = torch.empty(0, 32, device="cuda"), torch.full((32, 64), 5.0, device="cuda"), torch.full((32,), 5.0, device="cuda")
    pkg.esc_linear_forward(x, w, None, 0, out)
    pkg.esc_linear_backward(x, w, None, 0, out, torch.empty_like(x), gw, gb)
    assert (gw == 0).all() and (gb == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_same_bits(pkg, dtype):
    s = make(9001, 64, 128, dtype)
    runs = []
    for _ in range(3):
        got = [torch.empty_like(s["x"]), torch.empty_like(s["w"]), torch.empty_like(s["b"]), torch.empty_like(s["go"])]
        pkg.esc_linear_backward(s["x"], s["w"], s["z"], 2, s["go"], *got[:3])
        pkg.esc_linear_forward(s["x"], s["w"], s["b"], 2, got[3])
        runs.append(got)
    for r in runs[1:]:
        assert all(torch.equal(a, c) for a, c in zip(runs[0], r))
