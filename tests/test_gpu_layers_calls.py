"""Calls of the layer norm and of the linear layers as programs make them: other streams, several at once, captured and replayed, tensors of
more than 2^32 values, waits that run out."""
import threading
import time

import pytest
import torch

from tests import layers_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


class Layers:
    """A norm and a linear layer with their gradients, in tensors of their own."""

    def __init__(self, pkg, rows, C, N, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *n: torch.randn(*n, generator=g).to(dtype).cuda()   # noqa: E731
        self.pkg, self.x, self.w, self.b, self.W, self.B, self.go, self.z = pkg, rand(rows, C), rand(C), rand(C), rand(N, C), rand(N), rand(rows, N), rand(rows, N)
        new = torch.zeros_like
        self.y, self.out, self.zz = new(self.x), new(self.go), new(self.go)
        self.grads = [new(t) for t in (self.x, self.W, self.B, self.x, self.w, self.b)]
        self.ws = pkg.new_layer_norm_workspace(rows, C), pkg.new_linear_workspace(rows, C, N, pkg.ESC_ACT_GELU, dtype)

    def run(self, stream=None):
        p, (gx, gW, gB, gn, gw, gb) = self.pkg, self.grads
        p.esc_layer_norm_forward(self.x, self.w, self.b, 1e-6, self.y, stream=stream)
        p.esc_linear_forward(self.y, self.W, self.B, p.ESC_ACT_GELU, self.out, None, self.zz, stream=stream)
        p.esc_linear_backward(self.y, self.W, self.zz, p.ESC_ACT_GELU, self.go, gx, gW, gB, self.ws[1], stream=stream)
        p.esc_layer_norm_backward(self.x, self.w, 1e-6, gx, gn, gw, gb, self.x, self.ws[0], stream=stream)

    def results(self):
        return [t.clone() for t in (self.y, self.out, self.zz, *self.grads)]


SIZES = [(1000, 64, 96), (70, 250, 130), (5000, 128, 512)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", SIZES)
def test_streams_and_graphs(pkg, dtype, size):
    """The same bits on another stream, without a workspace of the caller's, and in a graph that is replayed with other inputs."""
    a = Layers(pkg, *size, dtype, 1)
    a.run()
    torch.cuda.synchronize()
    want = a.results()
    b = Layers(pkg, *size, dtype, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.run(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, b.results()))
    c = Layers(pkg, *size, dtype, 2)
    c.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for n in ("x", "w", "b", "W", "B", "go"):
        getattr(c, n).copy_(getattr(a, n))
    for t in (c.y, c.out, c.zz, *c.grads):
        t.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, c.results()))
    gx = torch.empty_like(a.y)
    pkg.esc_linear_backward(a.y, a.W, a.zz, 2, a.go, gx)
    assert torch.equal(gx, want[3])


def test_threads_and_streams_at_once(pkg):
    """Layers of several sizes and types on streams of their own, from threads of their own."""
    work = [Layers(pkg, *s, d, i) for i, (s, d) in enumerate((s, d) for s in SIZES for d in (torch.float32, torch.bfloat16))]
    for w in work:
        w.run()
    torch.cuda.synchronize()
    want = [w.results() for w in work]
    errors, start = [], threading.Barrier(len(work))

    def loop(w):
        try:
            torch.cuda.set_device(0)
            stream = torch.cuda.Stream()
            start.wait(30)
            for _ in range(100):
                w.run(stream)
            stream.synchronize()
        except Exception as e:   # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=loop, args=(w,)) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    torch.cuda.synchronize()
    assert not errors, errors
    for w, r in zip(work, want):
        assert all(torch.equal(p, q) for p, q in zip(r, w.results()))
    assert pkg.esc_linear_device_status() == 0


def test_launches(pkg):
    """A small bf16 layer's backward pass is one kernel and its sums."""
    s = Layers(pkg, 1000, 64, 128, torch.bfloat16, 3)
    pkg.esc_linear_backward(s.y, s.W, s.zz, 2, s.go, *s.grads[:3], s.ws[1])
    assert pkg.esc_convattn_last_launches() == 2
    pkg.esc_linear_forward(s.y, s.W, s.B, 2, s.out)
    assert pkg.esc_convattn_last_launches() == 1


def test_more_than_2_to_the_32_values(pkg):
    """The last rows of tensors whose offsets do not fit 32 bits."""
    free = torch.cuda.mem_get_info()[0]
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    rows, C = (1 << 32) // 1032 + 700, 1032
    x = torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(600, C, device="cuda").bfloat16()
    x[-600:] = tail
    w, b = torch.randn(C, device="cuda").bfloat16(), torch.randn(C, device="cuda").bfloat16()
    y = torch.empty_like(x)
    pkg.esc_layer_norm_forward(x, w, b, 1e-6, y)
    val, far = ref.norm(tail, w, b, 1e-6)
    ref.check("y", y[-600:], val, far)
    gx = torch.empty_like(x)
    gw, gb = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    pkg.esc_layer_norm_backward(x, w, 1e-6, x, gx, gw, gb)                 # rows of zeros have no gradient: the last rows alone count
    val, far = ref.norm(tail, w, None, 1e-6, tail)
    for n, t in (("gx", gx[-600:]), ("gw", gw), ("gb", gb)):
        ref.check(n, t, val, far)
    del x, y, gx
    rows, K, N = (1 << 32) // 64 + 1000, 16, 64
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(700, K, device="cuda").bfloat16()
    x[-700:] = tail
    W, B = torch.randn(N, K, device="cuda").bfloat16(), torch.randn(N, device="cuda").bfloat16()
    out = torch.empty(rows, N, dtype=torch.bfloat16, device="cuda")
    pkg.esc_linear_forward(x, W, B, 1, out)
    val, far = ref.linear(tail, W, B, "relu", None)
    ref.check("out", out[-700:], val, far)
    go = torch.zeros_like(out)
    go[-700:] = torch.randn(700, N, device="cuda").bfloat16()
    gx, gW, gB = torch.empty_like(x), torch.empty_like(W), torch.empty_like(B)
    for act, z in ((0, None), (1, out)):                                   # relu's slope from its result: the same sign
        pkg.esc_linear_backward(x, W, z, act, go, gx, gW, gB)
        val, far = ref.linear_grad(tail, W, None if z is None else z[-700:], "relu" if act else "none", go[-700:], True)
        for n, t in (("gx", gx[-700:]), ("gw", gW), ("gb", gB)):
            ref.check(n, t, val, far)
    assert (gx[:1000] == 0).all()


def test_a_wait_that_runs_out(pkg):
    assert pkg.esc_linear_device_status() == 0
    t0 = time.time()
    pkg.esc_linear_selftest_bounded_wait()
    assert pkg.esc_linear_device_status() == 8 and time.time() - t0 < 30
    assert pkg.esc_linear_device_status() == 0                             # once
    a = Layers(pkg, 300, 64, 64, torch.bfloat16, 4)                        # and the device goes on
    a.run()
    val, far = ref.linear(a.y, a.W, a.B, "gelu", None)
    ref.check("out", a.out, val, far)
    assert pkg.esc_linear_device_status() == 0


def test_status_is_refused_in_a_capture(pkg):
    graph, codes = torch.cuda.CUDAGraph(), []
    x = torch.zeros(4, device="cuda")
    with torch.cuda.graph(graph):
        x.add_(1)
        codes.append(pkg.esc_linear_device_status())
    assert codes == [3]


def test_refusals_of_the_binding(pkg):
    x, w = torch.zeros(8, 64, device="cuda"), torch.zeros(64, 64, device="cuda")
    out = torch.zeros(8, 64, device="cuda")
    for call in (lambda: pkg.esc_linear_forward(x, w.cpu(), None, 0, out), lambda: pkg.esc_linear_forward(x, w, None, 0, out, torch.zeros(8, 64)),
                 lambda: pkg.esc_linear_forward(x.double(), w.double(), None, 0, out.double())):
        with pytest.raises((ValueError, TypeError)):
            call()
    for call in (lambda: pkg.esc_linear_forward(x, w, None, 5, out), lambda: pkg.esc_linear_forward(x, w, None, 0, x), lambda: pkg.esc_linear_backward(x, w, None, 2, out, x.clone()),
                 lambda: pkg.esc_layer_norm_forward(x, None, None, -1.0, out), lambda: pkg.esc_layer_norm_forward(x, None, None, 1e-6, x),
                 lambda: pkg.esc_layer_norm_backward(x, None, 1e-6, out, torch.zeros_like(x), torch.zeros(64, device="cuda"))):
        with pytest.raises(pkg.EscError):
            call()
