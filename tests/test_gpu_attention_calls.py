"""Calls of the window attention and of the bias as a program with several threads and streams makes them."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def test_threads_with_windows_of_two_sizes(pkg):
    """Windows of 48 and of 32 pixels run the same kernels with different amounts of shared memory (94 and 53 KB forward): no thread's
    calls may take away what another's need.  Straight through the C entry, so that the threads are inside it at the same time."""
    heads, d, rounds = 1, 16, 4000
    g = torch.Generator().manual_seed(1)
    L, work = pkg.lib(), []
    for win in (48, 32, 48, 32):
        q, k, v = (torch.randn(1, win, win, heads * d, generator=g).to(torch.bfloat16).cuda() for _ in range(3))
        table = torch.randn((2 * win - 1) ** 2, heads, generator=g).to(torch.bfloat16).cuda()
        want, out, stream = torch.empty_like(q), torch.empty_like(q), torch.cuda.Stream()
        pkg.esc_window_attention_forward(q, k, v, heads, win, win, table, None, 0.25, want)
        args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), 1, heads, d, win, win, heads * d, win, win, table.data_ptr(), None, table.shape[0], 0.25,
                out.data_ptr(), None, pkg.ESC_BF16, stream.cuda_stream)
        work.append((args, want, out, (q, k, v, table, stream)))
    torch.cuda.synchronize()
    codes, start = [set() for _ in work], threading.Barrier(len(work))

    def loop(i):
        args = work[i][0]
        torch.cuda.set_device(0)
        start.wait(30)
        for _ in range(rounds):
            codes[i].add(L.esc_window_attention_forward(*args))

    threads = [threading.Thread(target=loop, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    torch.cuda.synchronize()
    assert all(c == {0} for c in codes), codes
    assert all(torch.equal(want, out) for _, want, out, _ in work)


def test_a_plan_over_slices_of_one_buffer(pkg):
    """Tensors that touch but do not overlap, and gradients that are one tensor, are a plan; a parameter of two names is not."""
    flat, g = torch.zeros(3000, device="cuda"), torch.ones(1000, device="cuda")
    m, v = torch.zeros(3000, device="cuda"), torch.zeros(3000, device="cuda")
    cut = lambda t: [t[i * 1000:(i + 1) * 1000] for i in range(3)]   # noqa: E731
    pkg.esc_adamw_step(pkg.new_adamw_plan(cut(flat), [g] * 3, cut(m), cut(v)), 1, 0.5, weight_decay=0.0)
    torch.cuda.synchronize()
    assert ((flat + 0.5).abs() <= 1e-6).all()                            # the first step is the gradient's sign: 0.5 / (1 + 1e-8)
    with pytest.raises(pkg.EscError):
        pkg.new_adamw_plan([flat[:1000], flat[500:1500]], [g] * 2, cut(m)[:2], cut(v)[:2])
    with pytest.raises(pkg.EscError):
        pkg.new_adamw_plan([flat[:1000]] * 2, [g] * 2, cut(m)[:2], cut(v)[:2])


class Blocks:
    """Where a call's own scratch lies in memory, and which blocks the current stream's pool hands out around it."""

    def __init__(self, monkeypatch, name):
        from paper_2503_06671_b200 import binding

        self.seen, plain = [], getattr(binding, name)

        def look(t):
            if t is not None and t.dtype == torch.uint8:
                self.seen.append((t.data_ptr(), t.numel()))
            return plain(t)

        monkeypatch.setattr(binding, name, look)

    def around(self, call, size, side):
        """`call` runs on `side`, which is busy for some time; the current stream has work pending on a block of that size that it has given back."""
        pending = torch.empty(size, dtype=torch.uint8, device="cuda")
        before = pending.data_ptr()
        torch.cuda._sleep(10_000_000)                                    # some 5 ms
        pending.fill_(1)
        del pending
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        call()
        after = [torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF) for _ in range(4)]
        torch.cuda.synchronize()
        (at, n), = self.seen
        assert n >= size
        assert not before <= at < before + size, "the call's scratch is memory that the current stream still writes"
        assert not any(t.data_ptr() <= at < t.data_ptr() + size for t in after), "the call's scratch went to the current stream while the call was pending"


def test_scratch_of_the_attention_on_another_stream(pkg, monkeypatch):
    """stream= alone, without making it the current one, and no workspace."""
    B, H, W, heads, d, win = 2, 64, 64, 2, 16, 16
    g = torch.Generator().manual_seed(2)
    q, k, v, go = (torch.randn(B, H, W, heads * d, generator=g).cuda() for _ in range(4))
    table = torch.randn((2 * win - 1) ** 2, heads, generator=g).cuda()
    out, lse, side = torch.empty_like(q), torch.empty(B, heads, H, W, device="cuda"), torch.cuda.Stream()
    pkg.esc_window_attention_forward(q, k, v, heads, win, win, table, None, 0.25, out, lse)
    grads = [[torch.zeros_like(q) for _ in range(3)] + [torch.zeros_like(table)] for _ in range(2)]
    size = pkg.esc_window_attention_backward_workspace_bytes(B, heads, d, H, W, win, win)
    pkg.esc_window_attention_backward(q, k, v, heads, win, win, table, None, 0.25, out, lse, go, *grads[0], pkg.new_window_attention_workspace(B, heads, d, H, W, win, win))
    torch.cuda.synchronize()
    Blocks(monkeypatch, "_address").around(
        lambda: pkg.esc_window_attention_backward(q, k, v, heads, win, win, table, None, 0.25, out, lse, go, *grads[1], stream=side), size, side)
    assert all(torch.equal(a, b) for a, b in zip(*grads))


def test_scratch_of_the_bias_on_another_stream(pkg, monkeypatch):
    heads, win = 2, 32
    grad = torch.randn(heads, win * win, win * win, device="cuda")
    tables, side = [torch.zeros((2 * win - 1) ** 2, heads, device="cuda") for _ in range(2)], torch.cuda.Stream()
    size = pkg.esc_relpos_bias_workspace_bytes(heads, win, win)
    pkg.esc_relpos_bias_backward(grad, None, win, win, tables[0], pkg.new_relpos_bias_workspace(heads, win, win))
    torch.cuda.synchronize()
    Blocks(monkeypatch, "_address").around(lambda: pkg.esc_relpos_bias_backward(grad, None, win, win, tables[1], stream=side), size, side)
    assert torch.equal(*tables)


def test_scratch_of_the_closing_convolution_on_another_stream(pkg, monkeypatch):
    B, C, H, W = 2, 64, 48, 40
    cat, go, w = torch.randn(B, H, W, C, device="cuda"), torch.randn(B, H, W, C, device="cuda"), torch.randn(C, C, device="cuda")
    got = [[torch.zeros_like(cat), torch.zeros(C, C, device="cuda"), torch.zeros(C, device="cuda")] for _ in range(2)]
    size, side = pkg.esc_conv_fuse_backward_workspace_bytes(B, C, H, W), torch.cuda.Stream()
    pkg.esc_conv_fuse_backward(cat, go, w, *got[0], pkg.ESC_NHWC, torch.empty(size, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    Blocks(monkeypatch, "_ptr").around(lambda: pkg.esc_conv_fuse_backward(cat, go, w, *got[1], pkg.ESC_NHWC, stream=side), size, side)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_stream_of_another_device_is_refused_before_anything_runs(pkg):
    """The check is made on the stream's own word, so a stand-in shows it on a machine with one GPU."""
    from paper_2503_06671_b200 import binding

    with pytest.raises(ValueError):
        binding._allocating_for(torch.cuda.current_stream(), torch.device("cuda", 1))


def test_a_plan_made_for_another_stream(pkg, monkeypatch):
    """The table of addresses is no memory that the current stream still writes: AdamW would write wherever that says."""
    p, g, m, v = (torch.zeros(5000, device="cuda") + (i == 1) for i in range(4))
    size, side, plans = pkg.esc_adamw_plan_bytes([5000]), torch.cuda.Stream(), []
    torch.cuda.synchronize()
    Blocks(monkeypatch, "_address").around(lambda: plans.append(pkg.new_adamw_plan([p], [g], [m], [v], stream=side)), size, side)
    pkg.esc_adamw_step(plans[0], 1, 0.5, weight_decay=0.0, stream=side)
    torch.cuda.synchronize()
    assert ((p + 0.5).abs() <= 1e-6).all()


def test_a_plan_dropped_behind_a_step_on_another_stream(pkg):
    """Its table is nobody else's until the step has read it, whatever stream the step runs on."""
    p, g, m, v = (torch.zeros(5000, device="cuda") + (i == 1) for i in range(4))
    size, side = pkg.esc_adamw_plan_bytes([5000]), torch.cuda.Stream()
    plan = pkg.new_adamw_plan([p], [g], [m], [v])
    at = plan.table.data_ptr()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    pkg.esc_adamw_step(plan, 1, 0.5, weight_decay=0.0, stream=side)
    del plan
    after = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(64)]   # not written: only where they lie is asked
    where = [t.data_ptr() for t in after]
    torch.cuda.synchronize()
    assert at not in where
    assert ((p + 0.5).abs() <= 1e-6).all()
