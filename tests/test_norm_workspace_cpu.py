"""The scratch of the layer norm's backward pass is what its kernels use: of rows that no block holds in registers few partial sums are kept."""
import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2503_06671_b200 import build, lib

    build.build()
    return lib()


@pytest.mark.parametrize("rows", [1, 592, 100000])
@pytest.mark.parametrize("C", [8193, 20000, 1 << 17, 1 << 20])
def test_long_rows_ask_for_what_they_use(L, rows, C):
    """256 columns to a block and four blocks an SM at most: no more than 592 x 256 columns of partial sums, or one of each, and three values a row."""
    sums = max(min(rows, 592) * 256 + C, C) * 2 * 4
    assert 0 < L.esc_layer_norm_backward_workspace_bytes(rows, C) <= sums + rows * 12 + 1024
