"""The operators as a training step uses them: the bias as a matrix and the attention that reads its table agree, the attention's gradients
go through AdamW into the projections' outputs and the table, eagerly and in one replayed graph."""
import math

import pytest
import torch

from tests import attention_ref as ref

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
B, H, W, HEADS, D, WH, WW = 2, 20, 27, 2, 16, 8, 12


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


class Block:
    """Packed q, k, v and the table as parameters (fp32, with the copies that the attention takes), their gradients and AdamW's states."""

    def __init__(self, pkg, dtype, eight, seed):
        g = torch.Generator().manual_seed(seed)
        self.pkg, self.dtype, C = pkg, DTYPES[dtype], HEADS * D
        offsets = (2 * WH - 1) * (2 * WW - 1)
        self.bucket = torch.randint(0, 23, (offsets,), generator=g, dtype=torch.int32).cuda()
        self.params = [torch.randn(B, H, W, 3 * C, generator=g).cuda(), torch.randn(23, HEADS, generator=g).cuda()]
        self.used = [p.to(self.dtype).clone() for p in self.params] if dtype == "bf16" else self.params
        self.grads = [torch.zeros_like(t) for t in self.used]
        self.go = torch.randn(B, H, W, C, generator=g).to(self.dtype).cuda()
        self.out, self.lse = torch.zeros_like(self.go), torch.zeros(B, HEADS, H, W, device="cuda")
        kind = torch.float8_e4m3fn if eight else torch.float32
        self.m, self.v = ([torch.zeros(p.shape, device="cuda").to(kind) for p in self.params] for _ in range(2))
        scales = [[torch.zeros(-(-p.numel() // 256), device="cuda") for p in self.params] for _ in range(2)] if eight else [None, None]
        self.plan = pkg.new_adamw_plan(self.params, self.grads, self.m, self.v, *scales, copies=self.used if dtype == "bf16" else None)
        self.ws = pkg.new_window_attention_workspace(B, HEADS, D, H, W, WH, WW)
        self.scalars = torch.zeros(4, device="cuda")

    def cut(self, t):
        C = HEADS * D
        return t[..., :C], t[..., C:2 * C], t[..., 2 * C:]

    def gradients(self):
        q, k, v = self.cut(self.used[0])
        self.pkg.esc_window_attention_forward(q, k, v, HEADS, WH, WW, self.used[1], self.bucket, 0.25, self.out, self.lse)
        self.pkg.esc_window_attention_backward(q, k, v, HEADS, WH, WW, self.used[1], self.bucket, 0.25, self.out, self.lse, self.go,
                                               *self.cut(self.grads[0]), self.grads[1], self.ws)

    def step(self):
        self.gradients()
        self.pkg.esc_adamw_step(self.plan, 1, 1e-2, scalars=self.scalars)

    def state(self):
        return [t.float() for t in (*self.params, *self.used, *self.grads, *self.m, *self.v, self.out, self.lse)]


@pytest.mark.parametrize("eight", [False, True], ids=["fp32", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_steps_eager_and_replayed(pkg, dtype, eight):
    a, b = Block(pkg, dtype, eight, 1), Block(pkg, dtype, eight, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        b.step()
    for t in range(1, 4):
        used = [x.float().cpu() for x in a.used]
        for x in (a, b):
            x.scalars.copy_(torch.tensor(pkg.esc_adamw_scalars(t, 1e-2, 0.9, 0.999, 0.01)))
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y)
        # this step's gradients are those of the parameters that it started from
        val, far = ref.attention(*a.cut(used[0]), HEADS, WH, WW, used[1], a.bucket.cpu(), 0.25, a.go.cpu(), dtype == "bf16")
        for n, t_ in zip(("g_q", "g_k", "g_v"), a.cut(a.grads[0])):
            ref.check(t_, val[n], far[n], n)
        ref.check(a.grads[1], val["g_table"], far["g_table"], "g_table")
        if dtype == "bf16":
            assert all(torch.equal(u, p.bfloat16()) for u, p in zip(a.used, a.params))
        assert all(torch.isfinite(p).all() for p in a.params)


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_matrix_is_the_bias_that_the_attention_adds(pkg, dtype):
    """One window: softmax(q k^T + the matrix) v in 64 bits, and the table's gradient through the matrix, are the attention's."""
    g = torch.Generator().manual_seed(7)
    n, C = WH * WW, HEADS * D
    offsets = (2 * WH - 1) * (2 * WW - 1)
    t = DTYPES[dtype]
    q, k, v, go = (torch.randn(1, WH, WW, C, generator=g).to(t).cuda() for _ in range(4))
    table = torch.randn(offsets, HEADS, generator=g).to(t).cuda()
    bias = pkg.esc_relpos_bias_forward(table, None, WH, WW, torch.empty(HEADS, n, n, dtype=t, device="cuda"))
    out, lse = torch.empty_like(q), torch.empty(1, HEADS, WH, WW, device="cuda")
    pkg.esc_window_attention_forward(q, k, v, HEADS, WH, WW, table, None, 0.25, out, lse)
    _, _, _, g_table = pkg.esc_window_attention_backward(q, k, v, HEADS, WH, WW, table, None, 0.25, out, lse, go, *(torch.empty_like(q) for _ in range(3)),
                                                         torch.empty_like(table))
    split = lambda x: x[0].double().reshape(n, HEADS, D).transpose(0, 1)   # noqa: E731
    p = torch.softmax(0.25 * split(q) @ split(k).transpose(1, 2) + bias.double(), 2)
    want = p @ split(v)
    _, far = ref.attention(*(x.cpu() for x in (q, k, v)), HEADS, WH, WW, table.cpu(), None, 0.25, go.cpu(), dtype == "bf16")
    ref.check(out, want.transpose(0, 1).reshape(1, WH, WW, C).cpu(), far["out"], "out")
    ds = p * (split(go) @ split(v).transpose(1, 2) - (split(go) * want).sum(2, keepdim=True))
    through = pkg.esc_relpos_bias_backward(ds.float(), None, WH, WW, torch.empty(offsets, HEADS, device="cuda"))
    terms = ref.table_grad(ds.abs().cpu(), offsets, ref.bucket_index(WH, WW, WH, WW, None))
    ref.check(g_table, through.double().cpu(), far["g_table"] + 1024 * ref.U * terms, "g_table")
    assert math.isfinite(float(lse.sum()))
