"""The forms of the window attention's kernels that maps of some size run (more queries to a warp or a thread, several staged tiles, blocks
with many windows), against the formulas in 64 bits on the device, within the bounds of attention_ref.  Each case says which
selections it is there for, and the test checks that its size still leads to them."""
import pytest
import torch

from tests import attention_ref as ref
from tests.test_gpu_window_attention import inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    import paper_2503_06671_b200 as p

    p.lib()
    return p


def sizes(shape):
    """(windows, tokens of the largest, padded channels, offsets)"""
    B, H, W, heads, d, wh, ww = shape
    return B * -(-H // wh) * -(-W // ww), min(wh, H) * min(ww, W), 16 if d <= 16 else 32 if d <= 32 else 64, (2 * wh - 1) * (2 * ww - 1)


def two_tiles(shape, sms):               # bf16 forward: 32 queries to a warp
    windows, tokens, D, _ = sizes(shape)
    return D <= 32 and windows * shape[3] * -(-tokens // 256) >= sms


def two_copies(shape, sms):              # bf16 forward: the head's table twice in shared memory
    _, _, D, _ = sizes(shape)
    return 4 * 128 * D * 2 + 3 * 128 * 12 + 2 * 4 * ((2 * shape[5] - 1) * 2 * shape[6] + 32) + 64 <= 112 * 1024


def odd_border(shape, sms):              # windows, or the last of a row, whose keys' bias is read one by one
    return (shape[2] % shape[6]) % 2 == 1 or shape[6] % 2 == 1


def full_tiles(shape, sms):              # more than one staged tile of 128 keys
    return sizes(shape)[1] > 128


def whole_pieces(shape, sms):            # rows that are copied 16 bytes at a time
    return shape[4] % 8 == 0


def listed_twice(shape, sms):            # bf16 table's gradient: more whole windows for a block than it lists at a time
    B, H, W, heads, d, wh, ww = shape
    tiles = -(-sizes(shape)[1] // 64)
    parts = min(max(1, 4 * sms // (heads * tiles)), -(-sizes(shape)[1] // 128))
    groups = max(1, 4 * sms // (heads * tiles * parts))
    return B * (H // wh) * (W // ww) > 64 * groups


def windows_in_turn(shape, sms):         # the same: more than one window for a block
    heads = shape[3]
    tiles = -(-sizes(shape)[1] // 64)
    parts = min(max(1, 4 * sms // (heads * tiles)), -(-sizes(shape)[1] // 128))
    return sizes(shape)[0] > max(1, 4 * sms // (heads * tiles * parts))


def two_queries(shape, sms):             # fp32 forward: two queries to a thread
    windows, tokens, D, _ = sizes(shape)
    return D <= 16 and windows * shape[3] * tokens >= 2 * 16 * 32 * sms


def units_in_turn(shape, sms):           # fp32 rows of queries: more than one tile of queries for a block, whatever the blocks of an SM (four at most)
    return sizes(shape)[0] > 4 * sms // shape[3]


CASES = [
    # B, H, W, heads, d, wh, ww
    ("bf16", (2, 96, 151, 4, 16, 32, 32), [two_tiles, two_copies, odd_border, full_tiles, whole_pieces]),
    ("bf16", (2, 96, 160, 4, 16, 32, 32), [two_tiles, two_copies, full_tiles, whole_pieces]),
    ("bf16", (1, 128, 256, 4, 16, 64, 64), [two_tiles, full_tiles, whole_pieces]),           # one copy: 64 x 64 leaves no room for two
    ("bf16", (1, 96, 149, 3, 32, 48, 48), [two_tiles, two_copies, odd_border, full_tiles, whole_pieces]),
    ("bf16", (1, 64, 192, 4, 32, 64, 64), [two_tiles, full_tiles, whole_pieces]),
    ("bf16", (3, 40, 50, 6, 30, 16, 16), [two_tiles, two_copies, full_tiles, windows_in_turn]),
    ("bf16", (2, 93, 155, 5, 16, 31, 31), [two_tiles, two_copies, odd_border, full_tiles, whole_pieces]),
    ("bf16", (4, 1, 4000, 4, 16, 1, 1000), [two_tiles, two_copies, full_tiles, whole_pieces]),
    ("bf16", (1, 1, 12000, 3, 16, 1, 8192), [two_tiles, full_tiles, whole_pieces]),
    ("bf16", (1, 72, 96, 2, 64, 24, 24), [full_tiles, whole_pieces, windows_in_turn]),
    ("bf16", (1, 104, 102, 64, 16, 4, 4), [two_tiles, listed_twice, whole_pieces]),
    ("bf16", (2, 96, 160, 16, 32, 8, 8), [two_tiles, windows_in_turn, whole_pieces]),
    ("bf16", (2, 96, 160, 8, 64, 8, 8), [windows_in_turn, whole_pieces]),
    ("fp32", (2, 96, 151, 5, 16, 32, 32), [two_queries]),
    ("fp32", (2, 100, 131, 8, 16, 24, 25), [two_queries]),
    ("fp32", (4, 120, 124, 8, 10, 7, 9), [two_queries, units_in_turn]),
    ("fp32", (1, 104, 102, 64, 16, 4, 4), [two_queries, units_in_turn]),
    ("fp32", (1, 64, 96, 16, 32, 8, 8), [units_in_turn]),
    ("fp32", (1, 64, 96, 16, 48, 8, 8), [units_in_turn]),
    ("fp32", (1, 1, 9000, 2, 24, 1, 4500), []),
]


def on_device(x, shape, scale, bf16):
    heads, wh, ww = shape[3], shape[5], shape[6]
    with torch.device("cuda"):
        val, far = ref.attention(*(x[n].cuda() for n in "qkv"), heads, wh, ww, x["table"].cuda(), None if x["bucket"] is None else x["bucket"].cuda(), scale,
                                 x["go"].cuda(), bf16)
    return val, far


@pytest.mark.parametrize("dtype,shape,reaches", CASES, ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v)) if isinstance(v, tuple) else "")
def test_attention(pkg, dtype, shape, reaches):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for f in reaches:
        assert f(shape, sms), f"{f.__name__}: this size does not lead there any more"
    buckets = "some" if shape[4] in (30, 24) else "offset"
    x = inputs(shape, dtype, sum(shape), buckets)
    scale = shape[4] ** -0.5
    got = run(pkg, x, shape, scale)
    val, far = on_device(x, shape, scale, dtype == "bf16")
    for n, t in got.items():
        ref.check(t, val[n].cpu(), far[n].cpu(), n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_copy_or_two_queries_with_masks(pkg, dtype):
    """Keys ahead of the query masked, in the kernels of large maps: rows of one key, a first staged tile that some rows have nothing of."""
    shape = (8, 1, 1500, 16, 16, 1, 750)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert (two_tiles if dtype == "bf16" else two_queries)(shape, sms)
    x = inputs(shape, dtype, 77)
    dx = torch.arange(-749, 750)                                         # query minus key
    x["table"][(dx < 0) | (dx > 300)] = -float("inf")                    # at most 300 places back, so a late row has none of the first keys
    got = run(pkg, x, shape, 0.25)
    val, far = on_device(x, shape, 0.25, dtype == "bf16")
    for n, t in got.items():
        ref.check(t, val[n].cpu(), far[n].cpu(), n)
