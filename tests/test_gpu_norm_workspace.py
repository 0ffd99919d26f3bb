"""Nothing is written behind the scratch of the layer norm's backward pass, where its kernels change and where its size does."""
import pytest
import torch

from tests import layers_ref as ref
from tests.test_gpu_layer_norm import make, pkg   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,C,pad", [(1, 64, 0), (2000, 64, 0), (700, 2047, 0), (700, 2049, 0), (700, 2050, 2), (700, 4096, 0), (700, 4104, 0), (700, 8192, 0), (700, 8192, 1),
                                        (1, 8193, 0), (700, 8193, 0), (700, 8200, 0), (640, 60000, 0), (3, 160000, 0)])
def test_nothing_behind_the_workspace(pkg, dtype, rows, C, pad):   # noqa: F811
    x, w, _, gy, skip = make(rows, C, dtype, pad)
    n = pkg.esc_layer_norm_backward_workspace_bytes(rows, C)
    ws = torch.full((n + 4096,), 123, dtype=torch.uint8, device="cuda")
    gx, gw, gb = torch.empty_like(gy), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    pkg.esc_layer_norm_backward(x, w, 1e-6, gy, gx, gw, gb, skip, ws[:n])
    assert (ws[n:] == 123).all()
    val, far = ref.norm(x, w, None, 1e-6, gy, skip)
    for name, t in (("gx", gx), ("gw", gw), ("gb", gb)):
        ref.check(name, t, val, far)
