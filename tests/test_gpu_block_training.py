"""The layers as a training step of the block uses them: norm, projection to q, k and v, window attention, projection with the residual, norm,
feed-forward network with the residual, and back, then AdamW; eagerly and in one replayed graph, against automatic differentiation in 64 bits.

Bounds: in fp32 each of some 20 operations is off by 1e-5 of its result's norm at most; in bf16 some 24 roundings of at most 2^-8 each lie between
an input and its gradient, which the residuals pass on without gain.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, H, W, HEADS, D, WIN, EPS = 2, 16, 24, 4, 16, 8, 1e-5
C, HIDDEN, TOKENS = HEADS * D, 2 * HEADS * D, WIN * WIN
NAMES = ["n1w", "n1b", "qkv", "qkvb", "table", "proj", "projb", "n2w", "n2b", "fc1", "fc1b", "fc2", "fc2b"]
SHAPES = [(C,), (C,), (3 * C, C), (3 * C,), ((2 * WIN - 1) ** 2, HEADS), (C, C), (C,), (C,), (C,), (HIDDEN, C), (HIDDEN,), (C, HIDDEN), (C,)]


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def parameters(seed):
    g = torch.Generator().manual_seed(seed)
    p = {}
    for n, s in zip(NAMES, SHAPES):
        t = torch.randn(*s, generator=g)
        p[n] = 1 + 0.2 * t if n in ("n1w", "n2w") else t * (s[1] ** -0.5 if len(s) == 2 and n != "table" else 0.2)
    return p, torch.randn(B, H, W, C, generator=g), torch.randn(B, H, W, C, generator=g)


class Block:
    def __init__(self, pkg, dtype, seed):
        self.pkg, self.dtype = pkg, dtype
        p, x, go = parameters(seed)
        self.master = {n: t.cuda().to(dtype).float() for n, t in p.items()}
        self.p = {n: t.to(dtype).clone() for n, t in self.master.items()} if dtype != torch.float32 else self.master
        self.x, self.go = x.to(dtype).cuda(), go.to(dtype).cuda()
        new = lambda width: torch.zeros(B, H, W, width, dtype=dtype, device="cuda")   # noqa: E731
        self.act = {n: new(w) for n, w in (("n1", C), ("qkv", 3 * C), ("att", C), ("mid", C), ("n2", C), ("z", HIDDEN), ("hid", HIDDEN), ("out", C))}
        self.lse = torch.zeros(B, HEADS, H, W, device="cuda")
        self.g = {n: torch.zeros_like(t) for n, t in self.p.items()}
        self.ga = {n: new(w) for n, w in (("hid", HIDDEN), ("n2", C), ("mid", C), ("att", C), ("qkv", 3 * C), ("n1", C), ("x", C))}
        rows = B * H * W
        self.ws_norm = pkg.new_layer_norm_workspace(rows, C)
        lin = lambda K, N, a: pkg.new_linear_workspace(rows, K, N, a, dtype)   # noqa: E731
        self.ws = {"qkv": lin(C, 3 * C, 0), "proj": lin(C, C, 0), "fc1": lin(C, HIDDEN, 2), "fc2": lin(HIDDEN, C, 0)}
        self.ws_att = pkg.new_window_attention_workspace(B, HEADS, D, H, W, WIN, WIN)
        m, v = ([torch.zeros_like(t) for t in self.master.values()] for _ in range(2))
        self.plan = pkg.new_adamw_plan(list(self.master.values()), list(self.g.values()), m, v, copies=list(self.p.values()) if dtype != torch.float32 else None)
        self.scalars = torch.tensor(pkg.esc_adamw_scalars(1, 1e-2, 0.9, 0.999, 0.01), device="cuda")

    def forward(self):
        e, p, a = self.pkg, self.p, self.act
        e.esc_layer_norm_forward(self.x, p["n1w"], p["n1b"], EPS, a["n1"])
        e.esc_linear_forward(a["n1"], p["qkv"], p["qkvb"], e.ESC_ACT_NONE, a["qkv"])
        q, k, v = (a["qkv"][..., i * C:(i + 1) * C] for i in range(3))
        e.esc_window_attention_forward(q, k, v, HEADS, WIN, WIN, p["table"], None, D ** -0.5, a["att"], self.lse)
        e.esc_linear_forward(a["att"], p["proj"], p["projb"], e.ESC_ACT_NONE, a["mid"], self.x)
        e.esc_layer_norm_forward(a["mid"], p["n2w"], p["n2b"], EPS, a["n2"])
        e.esc_linear_forward(a["n2"], p["fc1"], p["fc1b"], e.ESC_ACT_GELU, a["hid"], None, a["z"])
        e.esc_linear_forward(a["hid"], p["fc2"], p["fc2b"], e.ESC_ACT_NONE, a["out"], a["mid"])

    def backward(self):
        e, p, a, g, ga = self.pkg, self.p, self.act, self.g, self.ga
        e.esc_linear_backward(a["hid"], p["fc2"], None, e.ESC_ACT_NONE, self.go, ga["hid"], g["fc2"], g["fc2b"], self.ws["fc2"])
        e.esc_linear_backward(a["n2"], p["fc1"], a["z"], e.ESC_ACT_GELU, ga["hid"], ga["n2"], g["fc1"], g["fc1b"], self.ws["fc1"])
        e.esc_layer_norm_backward(a["mid"], p["n2w"], EPS, ga["n2"], ga["mid"], g["n2w"], g["n2b"], self.go, self.ws_norm)
        e.esc_linear_backward(a["att"], p["proj"], None, e.ESC_ACT_NONE, ga["mid"], ga["att"], g["proj"], g["projb"], self.ws["proj"])
        cut = lambda t: [t[..., i * C:(i + 1) * C] for i in range(3)]   # noqa: E731
        e.esc_window_attention_backward(*cut(a["qkv"]), HEADS, WIN, WIN, p["table"], None, D ** -0.5, a["att"], self.lse, ga["att"], *cut(ga["qkv"]), g["table"], self.ws_att)
        e.esc_linear_backward(a["n1"], p["qkv"], None, e.ESC_ACT_NONE, ga["qkv"], ga["n1"], g["qkv"], g["qkvb"], self.ws["qkv"])
        e.esc_layer_norm_backward(self.x, p["n1w"], EPS, ga["n1"], ga["x"], g["n1w"], g["n1b"], ga["mid"], self.ws_norm)

    def step(self):
        self.forward()
        self.backward()
        self.pkg.esc_adamw_step(self.plan, 1, 1e-2, scalars=self.scalars)


def exact(block):
    """(out, gradients by name, gradient of x) in 64 bits."""
    p = {n: t.detach().double().requires_grad_() for n, t in block.p.items()}
    x = block.x.double().requires_grad_()
    F = torch.nn.functional
    split = lambda t: t.reshape(B, H // WIN, WIN, W // WIN, WIN, HEADS, D).permute(0, 1, 3, 5, 2, 4, 6).reshape(-1, HEADS, TOKENS, D)   # noqa: E731
    q, k, v = (split(t) for t in F.linear(F.layer_norm(x, (C,), p["n1w"], p["n1b"], EPS), p["qkv"], p["qkvb"]).split(C, 3))
    i = torch.arange(TOKENS, device="cuda")
    at = (i[:, None] // WIN - i[None] // WIN + WIN - 1) * (2 * WIN - 1) + i[:, None] % WIN - i[None] % WIN + WIN - 1
    att = torch.softmax(q @ k.transpose(2, 3) * D ** -0.5 + p["table"][at].permute(2, 0, 1), 3) @ v
    att = att.reshape(B, H // WIN, W // WIN, HEADS, WIN, WIN, D).permute(0, 1, 4, 2, 5, 3, 6).reshape(B, H, W, C)
    mid = x + F.linear(att, p["proj"], p["projb"])
    out = mid + F.linear(F.gelu(F.linear(F.layer_norm(mid, (C,), p["n2w"], p["n2b"], EPS), p["fc1"], p["fc1b"])), p["fc2"], p["fc2b"])
    grads = torch.autograd.grad((out * block.go.double()).sum(), [*p.values(), x])
    return out.detach(), dict(zip(p, grads)), grads[-1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_the_block(pkg, dtype):
    b = Block(pkg, dtype, 1)
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    out, grads, gx = exact(b)
    rel = lambda a, e: float((a.double() - e).norm() / e.norm())   # noqa: E731
    bound = 2e-4 if dtype == torch.float32 else 24 * 2.0 ** -8
    far = {"out": rel(b.act["out"], out), "x": rel(b.ga["x"], gx), **{n: rel(b.g[n], grads[n]) for n in NAMES}}
    assert all(v <= bound for v in far.values()), far
    assert pkg.esc_linear_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_in_a_graph(pkg, dtype):
    """Three steps, eagerly and as a replayed graph: the same bits in every parameter."""
    a, b = Block(pkg, dtype, 2), Block(pkg, dtype, 2)
    for _ in range(3):
        a.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    before = {n: t.clone() for n, t in b.master.items()}
    with torch.cuda.graph(graph, stream=side):
        b.step()
    assert all(torch.equal(t, b.master[n]) for n, t in before.items())       # captured, not run
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for n in NAMES:
        assert torch.equal(a.master[n], b.master[n]) and torch.equal(a.p[n], b.p[n]), n
        assert torch.isfinite(a.master[n]).all() and not torch.equal(a.master[n], before[n]), n
