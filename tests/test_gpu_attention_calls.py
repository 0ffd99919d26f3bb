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
