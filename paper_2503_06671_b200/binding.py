"""ctypes binding with the same names as include/esc_convattn.h (argument marshalling only).

Tensors are torch CUDA tensors (or, for the *_host call, CPU tensors); the binding passes their
data pointers, the logical sizes and the current stream.  Logical shape is always [B,C,H,W]:
an NCHW call takes a contiguous [B,C,H,W] tensor, an NHWC call a contiguous [B,H,W,C] tensor.
"""
from __future__ import annotations

import contextlib
import ctypes
from pathlib import Path

ESC_F32, ESC_BF16 = 0, 1
ESC_NCHW, ESC_NHWC = 0, 1

_LIB_PATH = Path(__file__).resolve().parent / "lib" / "libesc_convattn.so"
_lib = None


class EscError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        text = esc_status_string(status)
        detail = esc_last_error() if self.status == 7 else ""
        super().__init__(f"{where}: status {self.status} ({text}){' -- ' + detail if detail else ''}")


def lib_path() -> Path:
    return _LIB_PATH


def lib():
    """The loaded C-ABI library; raises if it has not been built (no silent fall-back)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2503_06671_b200.build` "
                "(there is no CPU implementation to fall back to)")
        L = ctypes.CDLL(str(_LIB_PATH))
        vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.esc_convattn_forward.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, vp]
        L.esc_convattn_forward_ex.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_forward_fused.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_workspace_bytes.argtypes = [i, i, i, i, i]
        L.esc_convattn_workspace_bytes.restype = sz
        L.esc_convattn_workspace_init.argtypes = [vp, sz, vp]
        L.esc_convattn_dynkernel.argtypes = [vp, i, i, i, i, i, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_forward_mlp.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, i, vp, i, i, vp, sz, vp]
        L.esc_convattn_dynkernel_mlp.argtypes = [vp, i, i, i, i, i, vp, vp, vp, vp, i, vp, i, i, vp, sz, vp]
        L.esc_convattn_forward_pw.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_stencil_pw.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_forward_dense.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_stencil_dense.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_forward_variant.argtypes = [vp, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, i, vp, i, i, vp, sz, vp]
        L.esc_convattn_backward_workspace_bytes.argtypes = [i, i, i, i, i]
        L.esc_convattn_backward_workspace_bytes.restype = sz
        L.esc_convattn_backward.argtypes = [vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_backward_mlp.argtypes = [vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, i, vp, vp, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_backward_pw.argtypes = [vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_backward_dense_workspace_bytes.argtypes = [i, i, i, i, i]
        L.esc_convattn_backward_dense_workspace_bytes.restype = sz
        L.esc_convattn_backward_dense.argtypes = [vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_backward_variant.argtypes = [vp, vp, i, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, i, vp, vp, vp, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_conv_fuse_backward_workspace_bytes.argtypes = [i, i, i, i]
        L.esc_conv_fuse_backward_workspace_bytes.restype = sz
        L.esc_conv_fuse_backward.argtypes = [vp, vp, i, i, i, i, vp, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_dynkernel_static.argtypes = [vp, i, i, i, i, i, vp, vp, vp, i, i, vp]
        L.esc_convattn_stencil.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, i, i, vp, sz, vp]
        L.esc_convattn_forward_host.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, i, i]
        L.esc_convattn_device_status.argtypes = [vp, vp]
        L.esc_convattn_selftest_bounded_wait.argtypes = [vp, vp]
        L.esc_convattn_forward_host_submit.argtypes = [i, vp, i, i, i, i, i, i, vp, vp, vp, vp, i, i]
        L.esc_convattn_forward_host_wait.argtypes = [i]
        ll, f, dbl = ctypes.c_longlong, ctypes.c_float, ctypes.c_double
        L.esc_relpos_bias_forward.argtypes = [vp, vp, i, i, i, i, vp, i, vp]
        L.esc_relpos_bias_workspace_bytes.argtypes = [i, i, i]
        L.esc_relpos_bias_workspace_bytes.restype = sz
        L.esc_relpos_bias_backward.argtypes = [vp, vp, i, i, i, i, vp, i, vp, sz, vp]
        L.esc_window_attention_forward.argtypes = [vp, vp, vp, i, i, i, i, i, ll, i, i, vp, vp, i, f, vp, vp, i, vp]
        L.esc_window_attention_backward_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
        L.esc_window_attention_backward_workspace_bytes.restype = sz
        L.esc_window_attention_backward.argtypes = [vp, vp, vp, i, i, i, i, i, ll, i, i, vp, vp, i, f, vp, vp, vp, vp, vp, vp, vp, i, vp, sz, vp]
        L.esc_adamw_plan_bytes.argtypes = [i, vp]
        L.esc_adamw_plan_bytes.restype = sz
        L.esc_adamw_plan_init.argtypes = [i, vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, vp, sz, vp, vp]
        L.esc_adamw_step.argtypes = [vp, ll, i, i, i, ll, dbl, dbl, dbl, dbl, dbl, dbl, vp, vp, vp]
        L.esc_adamw_scalars.argtypes = [ll, dbl, dbl, dbl, dbl, dbl, vp]
        L.esc_convattn_set_tile_width.argtypes = [i]
        L.esc_convattn_set_stencil_engine.argtypes = [i]
        L.esc_convattn_set_fused_stage1.argtypes = [i]
        L.esc_convattn_set_dense_engine.argtypes = [i]
        L.esc_status_string.argtypes = [i]
        L.esc_status_string.restype = ctypes.c_char_p
        L.esc_last_error.restype = ctypes.c_char_p
        for name in ("esc_convattn_forward", "esc_convattn_forward_ex", "esc_convattn_forward_fused", "esc_convattn_workspace_init",
                     "esc_convattn_dynkernel", "esc_convattn_dynkernel_static", "esc_convattn_forward_mlp", "esc_convattn_dynkernel_mlp", "esc_convattn_forward_pw", "esc_convattn_stencil_pw", "esc_convattn_forward_dense", "esc_convattn_stencil_dense", "esc_convattn_forward_variant", "esc_convattn_backward", "esc_convattn_backward_mlp", "esc_convattn_backward_pw", "esc_convattn_backward_dense", "esc_convattn_backward_variant", "esc_conv_fuse_backward", "esc_convattn_stencil", "esc_convattn_forward_host", "esc_convattn_forward_host_submit", "esc_convattn_forward_host_wait",
                     "esc_relpos_bias_forward", "esc_relpos_bias_backward", "esc_window_attention_forward", "esc_window_attention_backward",
                     "esc_adamw_plan_init", "esc_adamw_step", "esc_adamw_scalars",
                     "esc_convattn_device_status", "esc_convattn_last_path", "esc_convattn_last_tile_width", "esc_convattn_set_tile_width", "esc_convattn_set_stencil_engine", "esc_convattn_set_fused_stage1", "esc_convattn_set_dense_engine", "esc_convattn_last_launches",
                     "esc_version"):
            getattr(L, name).restype = i
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    import torch

    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(status, where):
    if status != 0:
        raise EscError(status, where)


def _dtype_code(t):
    import torch

    if t.dtype == torch.float32:
        return ESC_F32
    if t.dtype == torch.bfloat16:
        return ESC_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dims(x, layout):
    if x.dim() != 4 or not x.is_contiguous():
        raise ValueError("x must be a contiguous 4-D tensor in the memory order named by `layout`")
    if layout == ESC_NCHW:
        B, C, H, W = x.shape
    elif layout == ESC_NHWC:
        B, H, W, C = x.shape
    else:
        raise ValueError("layout")
    return int(B), int(C), int(H), int(W)


def esc_status_string(status) -> str:
    return lib().esc_status_string(int(status)).decode()


def esc_last_error() -> str:
    return lib().esc_last_error().decode()


def esc_version() -> int:
    return lib().esc_version()


def esc_convattn_last_path() -> int:
    return lib().esc_convattn_last_path()


def esc_convattn_last_tile_width() -> int:
    return lib().esc_convattn_last_tile_width()


def esc_convattn_set_tile_width(tile_width: int) -> None:
    _check(lib().esc_convattn_set_tile_width(int(tile_width)), "esc_convattn_set_tile_width")


ESC_ENGINE_AUTO, ESC_ENGINE_FP32, ESC_ENGINE_TENSOR = 0, 1, 2


def esc_convattn_set_dense_engine(engine: int) -> None:
    _check(lib().esc_convattn_set_dense_engine(int(engine)), "esc_convattn_set_dense_engine")


def esc_convattn_set_fused_stage1(on: bool) -> None:
    _check(lib().esc_convattn_set_fused_stage1(1 if on else 0), "esc_convattn_set_fused_stage1")


def esc_convattn_set_stencil_engine(engine: int) -> None:
    _check(lib().esc_convattn_set_stencil_engine(int(engine)), "esc_convattn_set_stencil_engine")


def esc_convattn_last_launches() -> int:
    return lib().esc_convattn_last_launches()


def esc_convattn_workspace_bytes(B, C_a, H, W, K) -> int:
    return int(lib().esc_convattn_workspace_bytes(B, C_a, H, W, K))


def esc_convattn_workspace_init(workspace, stream=None):
    _check(lib().esc_convattn_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(),
                                             _stream(stream)), "esc_convattn_workspace_init")


def new_workspace(B, C_a, H, W, K, device="cuda"):
    """Allocate (with torch) and initialise a workspace for the calls that take one."""
    import torch

    n = esc_convattn_workspace_bytes(B, C_a, H, W, K)
    if n == 0:
        raise ValueError("invalid problem size")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    esc_convattn_workspace_init(ws)
    return ws


def esc_convattn_forward(x, C_a, K, w_large, w_dyn, b_dyn, out, stream=None):
    """fp32 NCHW forward (library-owned scratch).  x, out: contiguous [B,C,H,W] float32 CUDA tensors."""
    B, C, H, W = _dims(x, ESC_NCHW)
    _check(lib().esc_convattn_forward(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_dyn), _ptr(b_dyn),
                                      _ptr(out), _stream(stream)), "esc_convattn_forward")
    return out


def esc_convattn_forward_ex(x, C_a, K, w_large, w_dyn, b_dyn, out, layout, workspace, stream=None):
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_forward_ex(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_dyn), _ptr(b_dyn),
                                         _ptr(out), _dtype_code(x), layout, _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_forward_ex")
    return out


def esc_convattn_forward_fused(x, C_a, K, w_large, w_dyn, b_dyn, w_fuse, b_fuse, residual, out, layout, workspace, stream=None):
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_forward_fused(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_dyn), _ptr(b_dyn), _ptr(w_fuse),
                                            _ptr(b_fuse), _ptr(residual), _ptr(out), _dtype_code(x), layout, _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_forward_fused")
    return out


def esc_convattn_dynkernel(x, C_a, w_dyn, b_dyn, dk_out, layout, workspace, stream=None):
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_dynkernel(_ptr(x), B, C, C_a, H, W, _ptr(w_dyn), _ptr(b_dyn), _ptr(dk_out),
                                        _dtype_code(x), layout, _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_dynkernel")
    return dk_out


def esc_convattn_forward_mlp(x, C_a, K, w_large, w_down, b_down, w_up, b_up, out, layout, workspace, stream=None):
    """Forward pass with the two-layer kernel estimator (hidden width = w_down.shape[0])."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_forward_mlp(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_down), _ptr(b_down),
                                          _ptr(w_up), _ptr(b_up), int(w_down.shape[0]), _ptr(out), _dtype_code(x),
                                          layout, _ptr(workspace), workspace.numel() * workspace.element_size(),
                                          _stream(stream)),
           "esc_convattn_forward_mlp")
    return out


def esc_convattn_dynkernel_mlp(x, C_a, w_down, b_down, w_up, b_up, dk_out, layout, workspace, stream=None):
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_dynkernel_mlp(_ptr(x), B, C, C_a, H, W, _ptr(w_down), _ptr(b_down), _ptr(w_up),
                                            _ptr(b_up), int(w_down.shape[0]), _ptr(dk_out), _dtype_code(x), layout,
                                            _ptr(workspace), workspace.numel() * workspace.element_size(),
                                            _stream(stream)),
           "esc_convattn_dynkernel_mlp")
    return dk_out


def esc_convattn_forward_pw(x, C_a, K, w_large, w_point, w_dyn, b_dyn, out, layout, workspace, stream=None):
    """Forward pass in the decomposed form of Eq. 5: point-wise filter w_point [C_a,C_a], then the depth-wise stage."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_forward_pw(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_point), _ptr(w_dyn),
                                         _ptr(b_dyn), _ptr(out), _dtype_code(x), layout, _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_forward_pw")
    return out


def esc_convattn_stencil_pw(x, C_a, K, w_large, w_point, dk, out, layout, workspace=None, stream=None):
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_stencil_pw(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_point), _ptr(dk),
                                         _ptr(out), _dtype_code(x), layout, _ptr(workspace),
                                         0 if workspace is None else workspace.numel() * workspace.element_size(),
                                         _stream(stream)),
           "esc_convattn_stencil_pw")
    return out


def esc_convattn_forward_dense(x, C_a, K, w_dense, w_dyn, b_dyn, out, layout, workspace, stream=None):
    """Forward pass with the dense large kernel w_dense [C_a,C_a,K,K] (output channel, input channel, row, column)."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_forward_dense(_ptr(x), B, C, C_a, H, W, K, _ptr(w_dense), _ptr(w_dyn), _ptr(b_dyn),
                                            _ptr(out), _dtype_code(x), layout, _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_forward_dense")
    return out


def esc_convattn_stencil_dense(x, C_a, K, w_dense, dk, out, layout, workspace=None, stream=None):
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_stencil_dense(_ptr(x), B, C, C_a, H, W, K, _ptr(w_dense), _ptr(dk), _ptr(out),
                                            _dtype_code(x), layout, _ptr(workspace),
                                            0 if workspace is None else workspace.numel() * workspace.element_size(),
                                            _stream(stream)),
           "esc_convattn_stencil_dense")
    return out


ESC_LK_DEPTHWISE, ESC_LK_DECOMPOSED, ESC_LK_DENSE = 0, 1, 2


def esc_convattn_backward_workspace_bytes(B, C_a, H, W, K) -> int:
    return int(lib().esc_convattn_backward_workspace_bytes(B, C_a, H, W, K))


def new_backward_workspace(B, C_a, H, W, K, device="cuda"):
    """Allocate (with torch) and zero a workspace for esc_convattn_backward."""
    import torch

    n = esc_convattn_backward_workspace_bytes(B, C_a, H, W, K)
    if n == 0:
        raise ValueError("invalid problem size, or K is not odd in 3 .. 13")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    esc_convattn_workspace_init(ws)
    return ws


def esc_convattn_backward(x, grad_out, C_a, K, w_large, w_dyn, b_dyn, grad_x, grad_w_large, grad_w_dyn, grad_b_dyn,
                          layout, workspace, stream=None):
    """Gradients of esc_convattn_forward_ex: grad_x like x; the three weight gradients are fp32 tensors or None."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_backward(_ptr(x), _ptr(grad_out), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_dyn), _ptr(b_dyn),
                                       _ptr(grad_x), _ptr(grad_w_large), _ptr(grad_w_dyn), _ptr(grad_b_dyn),
                                       _dtype_code(x), layout, _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_backward")
    return grad_x


def esc_convattn_backward_mlp(x, grad_out, C_a, K, w_large, w_down, b_down, w_up, b_up, grad_x, grad_w_large, grad_w_down,
                              grad_b_down, grad_w_up, grad_b_up, layout, workspace, stream=None):
    """Gradients of esc_convattn_forward_mlp: grad_x like x; the five weight gradients are fp32 tensors or None."""
    B, C, H, W = _dims(x, layout)
    hidden = int(w_down.shape[0])
    _check(lib().esc_convattn_backward_mlp(_ptr(x), _ptr(grad_out), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_down), _ptr(b_down),
                                           _ptr(w_up), _ptr(b_up), hidden, _ptr(grad_x), _ptr(grad_w_large), _ptr(grad_w_down),
                                           _ptr(grad_b_down), _ptr(grad_w_up), _ptr(grad_b_up), _dtype_code(x), layout,
                                           _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_backward_mlp")
    return grad_x


def esc_convattn_backward_pw(x, grad_out, C_a, K, w_large, w_point, w_dyn, b_dyn, grad_x, grad_w_large, grad_w_point, grad_w_dyn,
                             grad_b_dyn, layout, workspace, stream=None):
    """Gradients of esc_convattn_forward_pw (decomposed form): grad_x like x; the four weight gradients are fp32 tensors or None."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_backward_pw(_ptr(x), _ptr(grad_out), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_point), _ptr(w_dyn),
                                          _ptr(b_dyn), _ptr(grad_x), _ptr(grad_w_large), _ptr(grad_w_point), _ptr(grad_w_dyn),
                                          _ptr(grad_b_dyn), _dtype_code(x), layout, _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_backward_pw")
    return grad_x


def esc_convattn_backward_dense_workspace_bytes(B, C_a, H, W, K) -> int:
    return int(lib().esc_convattn_backward_dense_workspace_bytes(B, C_a, H, W, K))


def new_backward_dense_workspace(B, C_a, H, W, K, device="cuda"):
    """Allocate (with torch) and zero a workspace for esc_convattn_backward_dense."""
    import torch

    n = esc_convattn_backward_dense_workspace_bytes(B, C_a, H, W, K)
    if n == 0:
        raise ValueError("invalid problem size, C_a is not 16, or K is not odd in 3 .. 13")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    esc_convattn_workspace_init(ws)
    return ws


def esc_convattn_backward_dense(x, grad_out, C_a, K, w_dense, w_dyn, b_dyn, grad_x, grad_w_dense, grad_w_dyn, grad_b_dyn, layout,
                                workspace, stream=None):
    """Gradients of esc_convattn_forward_dense: grad_x like x; the three weight gradients are fp32 tensors or None."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_backward_dense(_ptr(x), _ptr(grad_out), B, C, C_a, H, W, K, _ptr(w_dense), _ptr(w_dyn), _ptr(b_dyn),
                                             _ptr(grad_x), _ptr(grad_w_dense), _ptr(grad_w_dyn), _ptr(grad_b_dyn), _dtype_code(x),
                                             layout, _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_backward_dense")
    return grad_x


def esc_convattn_backward_variant(x, grad_out, C_a, K, large_kernel, w_large, w_point, w_down, b_down, w_up, b_up, grad_x,
                                  grad_w_large, grad_w_point, grad_w_down, grad_b_down, grad_w_up, grad_b_up, layout, workspace,
                                  stream=None):
    """Gradients of esc_convattn_forward_variant: any large-kernel form (ESC_LK_*) with either estimator (w_down None
    means one linear layer w_up, b_up).  Weight gradients are fp32 tensors or None."""
    B, C, H, W = _dims(x, layout)
    hidden = 0 if w_down is None else int(w_down.shape[0])
    _check(lib().esc_convattn_backward_variant(_ptr(x), _ptr(grad_out), B, C, C_a, H, W, K, int(large_kernel), _ptr(w_large),
                                               _ptr(w_point), _ptr(w_down), _ptr(b_down), _ptr(w_up), _ptr(b_up), hidden,
                                               _ptr(grad_x), _ptr(grad_w_large), _ptr(grad_w_point), _ptr(grad_w_down),
                                               _ptr(grad_b_down), _ptr(grad_w_up), _ptr(grad_b_up), _dtype_code(x), layout,
                                               _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_backward_variant")
    return grad_x


def esc_conv_fuse_backward_workspace_bytes(B, C, H, W) -> int:
    return int(lib().esc_conv_fuse_backward_workspace_bytes(B, C, H, W))


def esc_conv_fuse_backward(cat, grad_out, w_fuse, grad_cat, grad_w_fuse, grad_b_fuse, layout, workspace=None, stream=None):
    """Gradients of the closing 1x1 convolution: grad_cat like cat; grad_w_fuse [C,C] and grad_b_fuse [C] are fp32 tensors
    or None.  Without a workspace one is allocated with torch for the call."""
    import torch

    B, C, H, W = _dims(cat, layout)
    if workspace is None:
        n = esc_conv_fuse_backward_workspace_bytes(B, C, H, W)
        if n == 0:
            raise EscError(3, "esc_conv_fuse_backward_workspace_bytes")
        with _allocating_for(stream, cat.device):
            workspace = torch.empty(n, dtype=torch.uint8, device=cat.device)
    _check(lib().esc_conv_fuse_backward(_ptr(cat), _ptr(grad_out), B, C, H, W, _ptr(w_fuse), _ptr(grad_cat), _ptr(grad_w_fuse),
                                        _ptr(grad_b_fuse), _dtype_code(cat), layout, _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_conv_fuse_backward")
    return grad_cat


def esc_convattn_selftest_bounded_wait(workspace, stream=None):
    """Runs the library's bounded device-side wait on a barrier nothing signals (about a second): afterwards
    esc_convattn_device_status(workspace) returns 8 (ESC_DEV_TIMEOUT) once."""
    _check(lib().esc_convattn_selftest_bounded_wait(_ptr(workspace), _stream(stream)), "esc_convattn_selftest_bounded_wait")


def esc_convattn_forward_variant(x, C_a, K, large_kernel, w_large, w_point, w_down, b_down, w_up, b_up, out, layout,
                                 workspace, stream=None):
    """Any large-kernel form (ESC_LK_*) with either estimator: w_down None means one linear layer (w_up, b_up)."""
    B, C, H, W = _dims(x, layout)
    hidden = 0 if w_down is None else int(w_down.shape[0])
    _check(lib().esc_convattn_forward_variant(_ptr(x), B, C, C_a, H, W, K, int(large_kernel), _ptr(w_large), _ptr(w_point),
                                              _ptr(w_down), _ptr(b_down), _ptr(w_up), _ptr(b_up), hidden, _ptr(out),
                                              _dtype_code(x), layout, _ptr(workspace),
                                              workspace.numel() * workspace.element_size(), _stream(stream)),
           "esc_convattn_forward_variant")
    return out


def esc_convattn_dynkernel_static(x, C_a, w_dyn, b_dyn, dk_out, layout, stream=None):
    """Stage 1 without any device allocation: the scratch is a fixed array inside the library.

    For callers that may not call cudaMalloc (fixed-memory real-time loops, frameworks that own
    the allocator).  Limits and the sharing rule are in include/esc_convattn.h; sizes beyond the
    fixed scratch raise EscError with status 6."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_dynkernel_static(_ptr(x), B, C, C_a, H, W, _ptr(w_dyn), _ptr(b_dyn), _ptr(dk_out),
                                               _dtype_code(x), layout, _stream(stream)),
           "esc_convattn_dynkernel_static")
    return dk_out


def esc_convattn_stencil(x, C_a, K, w_large, dk, out, layout, workspace=None, stream=None):
    B, C, H, W = _dims(x, layout)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().esc_convattn_stencil(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(dk), _ptr(out),
                                      _dtype_code(x), layout, _ptr(workspace), nbytes, _stream(stream)),
           "esc_convattn_stencil")
    return out


def esc_convattn_forward_host(x, C_a, K, w_large, w_dyn, b_dyn, out, layout):
    """Host-buffer call: CPU tensors in, CPU tensor out; copies and synchronisation happen inside."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_forward_host(_ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_dyn), _ptr(b_dyn),
                                           _ptr(out), _dtype_code(x), layout), "esc_convattn_forward_host")
    return out


def esc_convattn_forward_host_submit(slot, x, C_a, K, w_large, w_dyn, b_dyn, out, layout):
    """Asynchronous half of the host-buffer call: enqueue on slot 0 or 1 and return.  The CPU tensors must be
    pinned and stay untouched until esc_convattn_forward_host_wait(slot) returns."""
    B, C, H, W = _dims(x, layout)
    _check(lib().esc_convattn_forward_host_submit(int(slot), _ptr(x), B, C, C_a, H, W, K, _ptr(w_large), _ptr(w_dyn),
                                                  _ptr(b_dyn), _ptr(out), _dtype_code(x), layout),
           "esc_convattn_forward_host_submit")


def esc_convattn_forward_host_wait(slot) -> None:
    _check(lib().esc_convattn_forward_host_wait(int(slot)), "esc_convattn_forward_host_wait")


def esc_convattn_device_status(workspace, stream=None) -> int:
    return lib().esc_convattn_device_status(_ptr(workspace), _stream(stream))


# ---- window self-attention, its relative position bias, AdamW ---------------------------------------------------------------


_HERE = contextlib.nullcontext()


def _address(t):
    return None if t is None else t.data_ptr()


def _stream_address(stream):
    import torch

    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _torch_stream(stream, device):
    import torch

    if stream is None:
        return torch.cuda.current_stream(device)
    return stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream.cuda_stream, device=device)


def _allocating_for(stream, device):
    """torch allocates for `stream` within: what a call on it uses for itself has to come from, and go back to, memory that this stream's
    order covers.  None: the current stream."""
    import torch

    if stream is None:
        return _HERE
    stream = _torch_stream(stream, device)
    if stream.device != device:
        raise ValueError(f"the stream of a call has to be of its tensors' device {device}, not of {stream.device}")
    return torch.cuda.stream(stream)


def _on_device(first, *others):
    """The tensors' one device, made current for the call that follows: kernels run where the data are."""
    import torch

    device = first.device
    for t in others:
        if t is not None and t.device != device:
            raise ValueError("the tensors of a call have to be on one CUDA device")
    if device.type != "cuda":
        raise ValueError("the tensors of a call have to be on a CUDA device")
    return _HERE if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _dense(name, t, shape, dtype):
    if t is None:
        return
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{name} has to be a contiguous {tuple(shape)} tensor of {dtype}, not {tuple(t.shape)} of {t.dtype}")


def _bucket_arg(bucket, win_h, win_w):
    if bucket is None:
        return
    import torch

    if bucket.numel() != (2 * win_h - 1) * (2 * win_w - 1) or bucket.dtype != torch.int32 or not bucket.is_contiguous():
        raise ValueError(f"bucket has to be a contiguous int32 tensor with an entry for each of the {(2 * win_h - 1) * (2 * win_w - 1)} offsets")


def esc_relpos_bias_forward(table, bucket, win_h, win_w, bias, stream=None):
    """bias [heads, N, N] (N = win_h win_w) from table [n_buckets, heads]; bucket: int32 bucket of every offset, or None."""
    n, heads = (int(x) for x in table.shape)
    _dense("table", table, (n, heads), table.dtype)
    _dense("bias", bias, (heads, win_h * win_w, win_h * win_w), table.dtype)
    _bucket_arg(bucket, win_h, win_w)
    with _on_device(table, bucket, bias):
        _check(lib().esc_relpos_bias_forward(_address(table), _address(bucket), n, heads, win_h, win_w, _address(bias), _dtype_code(table), _stream_address(stream)),
               "esc_relpos_bias_forward")
    return bias


def esc_relpos_bias_workspace_bytes(heads, win_h, win_w) -> int:
    return int(lib().esc_relpos_bias_workspace_bytes(heads, win_h, win_w))


def new_relpos_bias_workspace(heads, win_h, win_w, device="cuda"):
    import torch

    n = esc_relpos_bias_workspace_bytes(heads, win_h, win_w)
    if n == 0:
        raise ValueError("invalid window")
    return torch.empty(n, dtype=torch.uint8, device=device)


def esc_relpos_bias_backward(grad_bias, bucket, win_h, win_w, grad_table, workspace=None, stream=None):
    """grad_table [n_buckets, heads] fp32 from grad_bias [heads, N, N]."""
    import torch

    n, heads = (int(x) for x in grad_table.shape)
    _dense("grad_table", grad_table, (n, heads), torch.float32)
    _dense("grad_bias", grad_bias, (heads, win_h * win_w, win_h * win_w), grad_bias.dtype)
    _bucket_arg(bucket, win_h, win_w)
    with _on_device(grad_bias, bucket, grad_table, workspace):
        if workspace is None:
            with _allocating_for(stream, grad_bias.device):
                workspace = new_relpos_bias_workspace(heads, win_h, win_w)
        _check(lib().esc_relpos_bias_backward(_address(grad_bias), _address(bucket), n, heads, win_h, win_w, _address(grad_table), _dtype_code(grad_bias),
                                              _address(workspace), workspace.numel() * workspace.element_size(), _stream_address(stream)),
               "esc_relpos_bias_backward")
    return grad_table


def _pixel_step(t):
    """Values between neighbouring pixels of a map [B, H, W, C]; ValueError where they are not evenly spaced, or dense in their channels."""
    B, H, W, C = t.shape
    b, h, w, c = t.stride()
    step = w if W > 1 else h if H > 1 else b if B > 1 else C                # from the innermost axis that has more than one entry
    if (C > 1 and c != 1) or (W > 1 and w != step) or (H > 1 and h != step * W) or (B > 1 and b != step * W * H):
        raise ValueError("pixels have to be dense in their channels and evenly spaced")
    return step


def _pixels(heads, first, *others):
    """(B, H, W, head_dim, pixel stride) of maps [B, H, W, heads * head_dim] that are laid out alike."""
    shape, strides, dtype = first.shape, first.stride(), first.dtype
    if len(shape) != 4 or heads < 1 or shape[3] % heads != 0:
        raise ValueError("the maps have to be [B, H, W, heads * head_dim]")
    step = _pixel_step(first)
    for t in others:
        if t.shape != shape or t.dtype != dtype or (t.stride() != strides and _pixel_step(t) != step):
            raise ValueError("q, k, v and their gradients have to be of one shape and type, with pixels alike")
    B, H, W, C = shape
    return B, H, W, C // heads, step


def esc_window_attention_forward(q, k, v, heads, win_h, win_w, table, bucket, scale, out, lse=None, stream=None):
    """out [B, H, W, heads * head_dim] (and lse [B, heads, H, W] fp32) of the self-attention over windows.

    q, k, v: [B, H, W, heads * head_dim], of their own or slices along the last axis of one packed tensor; table
    [n_buckets, heads] with the bucket of every offset (None: one row per offset), or None for no bias."""
    import torch

    B, H, W, d, step = _pixels(heads, q, k, v)
    _dense("out", out, (B, H, W, heads * d), q.dtype)
    _dense("lse", lse, (B, heads, H, W), torch.float32)
    n = 0 if table is None else int(table.shape[0])
    _dense("table", table, (n, heads), q.dtype)
    _bucket_arg(bucket, win_h, win_w)
    with _on_device(q, k, v, table, bucket, out, lse):
        _check(lib().esc_window_attention_forward(_address(q), _address(k), _address(v), B, heads, d, H, W, step, win_h, win_w, _address(table), _address(bucket), n, scale,
                                                  _address(out), _address(lse), _dtype_code(q), _stream_address(stream)),
               "esc_window_attention_forward")
    return out


def esc_window_attention_backward_workspace_bytes(B, heads, head_dim, H, W, win_h, win_w) -> int:
    return int(lib().esc_window_attention_backward_workspace_bytes(B, heads, head_dim, H, W, win_h, win_w))


def new_window_attention_workspace(B, heads, head_dim, H, W, win_h, win_w, device="cuda"):
    """Scratch of esc_window_attention_backward."""
    import torch

    n = esc_window_attention_backward_workspace_bytes(B, heads, head_dim, H, W, win_h, win_w)
    if n == 0:
        raise ValueError("invalid problem size")
    return torch.empty(n, dtype=torch.uint8, device=device)


def esc_window_attention_backward(q, k, v, heads, win_h, win_w, table, bucket, scale, out, lse, grad_out, grad_q, grad_k, grad_v, grad_table=None,
                                  workspace=None, stream=None):
    """Gradients of esc_window_attention_forward; grad_q, grad_k, grad_v are laid out like q, k, v."""
    import torch

    B, H, W, d, step = _pixels(heads, q, k, v, grad_q, grad_k, grad_v)
    _dense("out", out, (B, H, W, heads * d), q.dtype)
    _dense("grad_out", grad_out, (B, H, W, heads * d), q.dtype)
    _dense("lse", lse, (B, heads, H, W), torch.float32)
    n = 0 if table is None else int(table.shape[0])
    _dense("table", table, (n, heads), q.dtype)
    _dense("grad_table", grad_table, (n, heads), q.dtype)
    _bucket_arg(bucket, win_h, win_w)
    with _on_device(q, k, v, table, bucket, out, lse, grad_out, grad_q, grad_k, grad_v, grad_table, workspace):
        if workspace is None:
            with _allocating_for(stream, q.device):
                workspace = new_window_attention_workspace(B, heads, d, H, W, win_h, win_w)
        _check(lib().esc_window_attention_backward(_address(q), _address(k), _address(v), B, heads, d, H, W, step, win_h, win_w, _address(table), _address(bucket), n, scale,
                                                   _address(out), _address(lse), _address(grad_out), _address(grad_q), _address(grad_k), _address(grad_v), _address(grad_table),
                                                   _dtype_code(q), _address(workspace), workspace.numel() * workspace.element_size(), _stream_address(stream)),
               "esc_window_attention_backward")
    return grad_q, grad_k, grad_v, grad_table


ESC_STATES_F32, ESC_STATES_E4M3 = 0, 1
ADAMW_QUANT = 256   # values of a tensor that share a scale with ESC_STATES_E4M3


def esc_adamw_plan_bytes(sizes) -> int:
    return int(lib().esc_adamw_plan_bytes(len(sizes), (ctypes.c_longlong * len(sizes))(*sizes)))


class AdamwPlan:
    """A list of tensors in device memory, as esc_adamw_step takes it.  It keeps the tensors.  A graph that has captured its steps needs it as
    long as it is replayed."""

    def __init__(self, table, n_chunks, param_dtype, grad_dtype, states, tensors, stream=None):
        self.table, self.n_chunks, self.param_dtype, self.grad_dtype, self.states, self.tensors = table, n_chunks, param_dtype, grad_dtype, states, tensors
        self.stream = stream   # address of the stream that the table was allocated for


def esc_adamw_plan_init(params, grads, exp_avgs, exp_avg_sqs, avg_scales=None, sq_scales=None, copies=None, stream=None):
    """The plan of a list of tensors: parameters and gradients of fp32 or bf16, states of fp32, or of float8_e4m3fn with fp32 scales
    of ceil(size / 256) entries (exp_avg_sqs then holds the square roots); copies (bf16) and single entries of it may be None."""
    import torch

    n = len(params)
    if n == 0 or not (n == len(grads) == len(exp_avgs) == len(exp_avg_sqs)) or any(x is not None and len(x) != n for x in (avg_scales, sq_scales, copies)):
        raise ValueError("the lists have to be as long as one another, and not empty")
    p, g, s = params[0].dtype, grads[0].dtype, exp_avgs[0].dtype
    eight = s == torch.float8_e4m3fn
    if not eight and s != torch.float32:
        raise TypeError(f"unsupported dtype {s} of the states")
    if eight != (avg_scales is not None) or eight != (sq_scales is not None):
        raise ValueError("states in 8 bits have scales, others have none")
    sizes = [t.numel() for t in params]

    def pointers(name, tensors, dtype, counts):
        if tensors is None:
            return None
        for t, count in zip(tensors, counts):
            if t is not None and (t.numel() != count or t.dtype != dtype or not t.is_contiguous()):
                raise ValueError(f"{name}: contiguous tensors of {dtype}, as many values as the parameters (scales: one for 256)")
        return (ctypes.c_void_p * n)(*[t.data_ptr() if t is not None and t.numel() else None for t in tensors])

    scales = [-(-k // ADAMW_QUANT) for k in sizes]
    lists = [("params", params, p, sizes), ("grads", grads, g, sizes), ("exp_avgs", exp_avgs, s, sizes), ("exp_avg_sqs", exp_avg_sqs, s, sizes),
             ("avg_scales", avg_scales, torch.float32, scales), ("sq_scales", sq_scales, torch.float32, scales), ("copies", copies, torch.bfloat16, sizes)]
    every = [t for _, ts, _, _ in lists if ts is not None for t in ts if t is not None]
    arrays = [pointers(*x) for x in lists]
    states = ESC_STATES_E4M3 if eight else ESC_STATES_F32
    chunks = ctypes.c_longlong()
    with _on_device(*every):
        bytes_ = esc_adamw_plan_bytes(sizes)
        if bytes_ == 0:
            raise ValueError("invalid sizes")
        with _allocating_for(stream, params[0].device):                 # the copy of the addresses waits for nobody else's work
            table = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
        _check(lib().esc_adamw_plan_init(n, (ctypes.c_longlong * n)(*sizes), *arrays, _dtype_code(params[0]), _dtype_code(grads[0]), states, _address(table), bytes_,
                                         ctypes.byref(chunks), _stream_address(stream)), "esc_adamw_plan_init")
        at = _stream_address(stream)
    return AdamwPlan(table, chunks.value, _dtype_code(params[0]), _dtype_code(grads[0]), states, every, at)


new_adamw_plan = esc_adamw_plan_init


def esc_adamw_scalars(step, lr, beta1, beta2, weight_decay, grad_scale=1.0):
    """The four numbers that a `scalars` tensor of esc_adamw_step holds."""
    out = (ctypes.c_float * 4)()
    _check(lib().esc_adamw_scalars(int(step), lr, beta1, beta2, weight_decay, grad_scale, out), "esc_adamw_scalars")
    return list(out)


def esc_adamw_step(plan, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0, scalars=None, skip=None, stream=None):
    """One AdamW step over the plan's tensors.  scalars (4 fp32 on the device, from esc_adamw_scalars) replaces step, lr, weight_decay and
    grad_scale, for captured graphs; skip: an int32 on the device, not zero: the call changes nothing."""
    import torch

    _dense("scalars", scalars, (4,), torch.float32)
    if skip is not None and (skip.numel() != 1 or skip.dtype != torch.int32):
        raise ValueError("skip has to be one int32")
    with _on_device(plan.table, scalars, skip):
        at = _stream_address(stream)
        if at != plan.stream:                                           # a plan that is dropped keeps its memory until this step is over
            plan.table.record_stream(_torch_stream(stream, plan.table.device))
        _check(lib().esc_adamw_step(_address(plan.table), plan.n_chunks, plan.param_dtype, plan.grad_dtype, plan.states, int(step), lr, beta1, beta2, eps,
                                    weight_decay, grad_scale, _address(scalars), _address(skip), at), "esc_adamw_step")
