"""What the attention, bias and AdamW entry points do on the host at the ends of their ranges, before anything could be launched."""
import ctypes

import pytest

UNSUPPORTED = 3
Q, K, V, O, T = (0x10000000000 * i for i in range(1, 6))   # never dereferenced


@pytest.fixture(scope="module")
def L():
    from paper_2503_06671_b200 import build, lib

    build.build()
    return lib()


def test_maps_as_high_as_an_int_can_say(L):
    """One column of 2^31 - 1 pixels: the number of windows is rounded up without leaving 32 bits on the way."""
    size = L.esc_window_attention_backward_workspace_bytes
    rows = 2 ** 31 - 1
    assert size(1, 1, 1, rows, 1, 2, 1) == size(1, 1, 1, rows, 1, 1, 1) == 0           # 2^30 and 2^31 windows: more than 1e9 blocks
    assert 2 * 4 * rows <= size(1, 1, 1, rows, 1, 64, 1) <= 2 * 4 * rows + (64 << 20)   # two fp32 values a row, and the table's sums
    fwd = lambda wh: L.esc_window_attention_forward(Q, K, V, 1, 1, 1, rows, 1, 1, wh, 1, T, None, 2 * wh - 1, 1.0, O, None, 1, None)   # noqa: E731
    assert fwd(1) == fwd(2) == UNSUPPORTED


def test_more_buckets_than_the_kernels_can_number(L):
    """The kernels count buckets by 32 in an int; a table of more than 2^30 rows is refused."""
    B, WS, many = 0x60000000000, 0x70000000000, 2 ** 30 + 1
    for n in (many, 2 ** 31 - 1):
        assert L.esc_relpos_bias_forward(T, B, n, 1, 2, 2, O, 0, None) == UNSUPPORTED
        assert L.esc_relpos_bias_backward(O, B, n, 1, 2, 2, T, 0, WS, 1 << 20, None) == UNSUPPORTED
        assert L.esc_window_attention_forward(Q, K, V, 1, 1, 1, 4, 4, 1, 2, 2, T, B, n, 1.0, O, None, 1, None) == UNSUPPORTED


def test_adamw_plans_with_a_tensor_twice(L):
    """A parameter of two names, states that overlap, a copy over its own parameter, a plan inside a tensor: two threads would change one value."""
    ALIAS, n = 5, ctypes.c_longlong()
    sizes = (ctypes.c_longlong * 3)(1000, 0, 5000)
    names = dict(p=0x10000000, g=0x20000000, m=0x30000000, v=0x40000000, ms=0x50000000, vs=0x60000000, c=0x70000000)

    def init(eight=False, plan=0x80000000, **other):
        lists = {k: [base, None, base + 0x100000] for k, base in names.items()}
        for k, (i, at) in other.items():
            lists[k][i] = at
        arr = {k: (ctypes.c_void_p * 3)(*x) for k, x in lists.items()}
        return L.esc_adamw_plan_init(3, sizes, arr["p"], arr["g"], arr["m"], arr["v"], arr["ms"] if eight else None, arr["vs"] if eight else None, arr["c"],
                                     0, 0, int(eight), plan, 1 << 20, ctypes.byref(n), None)

    assert init(p=(2, names["p"])) == init(p=(2, names["p"] + 3996)) == init(m=(2, names["m"])) == init(v=(0, names["m"])) == ALIAS
    assert init(c=(0, names["p"])) == init(c=(2, names["c"] + 1996)) == init(g=(2, names["p"] + 16)) == init(m=(0, names["g"] + 0x100000 + 19996)) == ALIAS
    assert init(True, ms=(2, names["ms"] + 12)) == init(True, vs=(0, names["ms"])) == init(True, m=(2, names["m"] + 996)) == ALIAS
    assert init(plan=names["v"] + 256) == init(plan=names["p"]) == ALIAS   # four runs of 64 bytes
