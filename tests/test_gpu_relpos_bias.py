"""The relative position bias as a matrix and the gradient of its table, against the formulas in 64 bits.

The matrix is a copy: equal bits.  The gradient is a sum of n terms in fp32 in a fixed tree: at most n + 8 roundings of 2^-24 of the
terms' magnitudes; the trees are at most 64 + 32 + 32 + 512 long, so 1024 u bounds them."""
import pytest
import torch

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
WINDOWS = [(1, 1), (1, 2), (3, 1), (2, 3), (8, 8), (7, 9), (5, 16), (16, 17), (24, 24), (32, 32), (3, 40), (1, 257), (1, 1000), (100, 1), (64, 64)]


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def case(wh, ww, heads, dtype, buckets, seed):
    g = torch.Generator().manual_seed(seed)
    offsets = (2 * wh - 1) * (2 * ww - 1)
    bucket, n = None, offsets
    if buckets:
        n = buckets
        bucket = torch.randint(0, n, (offsets,), generator=g, dtype=torch.int32)
        bucket[::7] = -3
        bucket[3::11] = n
    return torch.randn(n, heads, generator=g).to(DTYPES[dtype]), bucket, g


@pytest.mark.parametrize("buckets", [0, 1, 37, 700])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", WINDOWS, ids=lambda w: "%dx%d" % w)
def test_bias(pkg, window, dtype, buckets):
    wh, ww = window
    n = wh * ww
    heads = 1 if n > 1000 else 3
    table, bucket, g = case(wh, ww, heads, dtype, buckets, n + buckets)
    dev = bucket.cuda() if bucket is not None else None
    room = torch.full((heads * n * n + 16,), 9.0, dtype=DTYPES[dtype], device="cuda")
    bias = room[:heads * n * n].view(heads, n, n)
    pkg.esc_relpos_bias_forward(table.cuda(), dev, wh, ww, bias)
    if n <= 1100:
        assert torch.equal(bias.cpu().double(), ref.bias_matrix(table, bucket, wh, ww))
    else:                                                                # the same in pieces, on the device
        at = ref.bucket_index(wh, ww, wh, ww, bucket).cuda()
        t = table.cuda()
        for h in range(heads):
            want = torch.where((at >= 0) & (at < t.shape[0]), t[:, h][at.clamp(0, t.shape[0] - 1)], torch.zeros((), dtype=t.dtype, device="cuda"))
            assert torch.equal(bias[h], want)
    assert (room[heads * n * n:] == 9.0).all()
    grad = torch.randn(heads, n, n, generator=g).to(DTYPES[dtype])
    g_table = torch.full((table.shape[0], heads), float("nan"), device="cuda")
    ws = pkg.new_relpos_bias_workspace(heads, wh, ww)
    ws.fill_(0xFF)
    pkg.esc_relpos_bias_backward(grad.cuda(), dev, wh, ww, g_table, ws)
    again = torch.empty_like(g_table)
    pkg.esc_relpos_bias_backward(grad.cuda(), dev, wh, ww, again, ws)
    at = ref.bucket_index(wh, ww, wh, ww, bucket)
    ref.check(g_table, ref.table_grad(grad, table.shape[0], at), 1024 * ref.U * ref.table_grad(grad.abs(), table.shape[0], at) + 1e-37, "g_table")
    assert torch.equal(g_table, again)


def test_infinities_pass(pkg):
    table = torch.randn(15 * 15, 2, device="cuda")
    table[7], table[100] = -float("inf"), float("nan")
    bias = torch.empty(2, 64, 64, device="cuda")
    pkg.esc_relpos_bias_forward(table, None, 8, 8, bias)
    want = table.t()[:, ref.bucket_index(8, 8, 8, 8, None).cuda()]
    assert torch.equal(torch.nan_to_num(bias, nan=123.0), torch.nan_to_num(want, nan=123.0))


def test_captured_on_a_side_stream(pkg):
    table, bucket, g = case(12, 12, 2, "bf16", 19, 4)
    t, b = table.cuda(), bucket.cuda()
    bias = torch.empty(2, 144, 144, dtype=torch.bfloat16, device="cuda")
    g_table = torch.zeros(19, 2, device="cuda")
    ws = pkg.new_relpos_bias_workspace(2, 12, 12)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        pkg.esc_relpos_bias_forward(t, b, 12, 12, bias)
        pkg.esc_relpos_bias_backward(bias, b, 12, 12, g_table, ws)
    t.mul_(2)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    want = ref.bias_matrix(t.cpu(), bucket, 12, 12)
    assert torch.equal(bias.cpu().double(), want)
    at = ref.bucket_index(12, 12, 12, 12, bucket)
    ref.check(g_table, ref.table_grad(want, 19, at), 1024 * ref.U * ref.table_grad(want.abs(), 19, at) + 1e-37, "g_table")


def test_refuses(pkg):
    table, bias = torch.zeros(9, 2, device="cuda"), torch.zeros(2, 4, 4, device="cuda")
    pkg.esc_relpos_bias_forward(table, None, 2, 2, bias)
    with pytest.raises(pkg.EscError):
        pkg.esc_relpos_bias_forward(table[:8].contiguous(), None, 2, 2, bias)
    with pytest.raises(ValueError):
        pkg.esc_relpos_bias_forward(table, None, 2, 2, bias.bfloat16())
    with pytest.raises(ValueError):
        pkg.esc_relpos_bias_forward(table, torch.zeros(9, dtype=torch.int64, device="cuda"), 2, 2, bias)
    with pytest.raises(pkg.EscError):
        pkg.esc_relpos_bias_backward(bias, None, 2, 2, torch.zeros(9, 2, device="cuda"), torch.zeros(16, dtype=torch.uint8, device="cuda"))
