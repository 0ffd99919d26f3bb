"""Layer norm and linear layers in 64 bits, as the formulas stand, with bounds for what the kernels may be off.

Bounds: u = 2^-24 (half a step of fp32) for every fp32 operation, h = 2^-8 (bf16, half a step) for every rounding to bf16, first order; a
sum of n terms is off by n u of the sum of magnitudes whatever its order, by twice that where the tensor cores may truncate; functions of
CUDA's library by the steps that its documentation states (erfc 4, exp 2, rsqrt 2 steps of 2 u each).
  norm     e_mu = (n + 2) u mean|x|;  e_d = e_mu + u |d|;  var: (n + 3) u var + 2 e_mu mean|d| + e_mu^2;  r: relative rho = half of that / (var + eps) + 5 u
           y: |w| (r e_d + |d| r (rho + 3 u)) + u |y| + u |b|;   xh: e_x = r e_d + |xh| (rho + u)
           gx: r (u |a| + (n + 2) u mean|a| + |xh| e_al + |al| e_x + 4 u (|a| + |mean a| + |xh al|)) + rho |gx - skip| + u (|gx| + |skip|),
           e_al = (n + 4) u mean|a xh| + mean(|a| e_x);   gw: (rows + 2) u sum |gy xh| + sum |gy| e_x;   gb: rows u sum |gy|
  linear   e_z = 2 (K + 2) u (sum |x w| + |b|);  act: its slope (1.13 at most) e_z + 12 u |act|;  out: + u (|act| + |residual|)
           slope: e_s = 8 u Phi + (z^2 + 8) u |z phi|;  e_g = |go| e_s + u |g|;  bf16 with an activation: + h |g| (an operand of two products, not of gb)
           gx: sum e_g |w| + 2 (N + 2) u sum |g w|;  gw: sum e_g |x| + 2 (rows + 2) u sum |g x|;  gb: sum e_g + 2 (rows + 2) u sum |g|
and h of the result where it is bf16.
"""
import math

import torch

U, H8 = 2.0 ** -24, 2.0 ** -8
FLOOR = 1e-37                                                           # below the normal numbers


def norm(x, w, b, eps, gy=None, skip=None):
    """({name: value}, {name: bound without the rounding to bf16}) of y, or of gx, gw, gb; tensors [rows, C]."""
    x = x.double()
    n, rows = x.shape[1], x.shape[0]
    w = torch.ones(n, dtype=torch.float64, device=x.device) if w is None else w.double()
    mean = lambda t: t.mean(1, keepdim=True)   # noqa: E731
    d = x - mean(x)
    var = mean(d * d)
    r = (var + eps) ** -0.5
    xh = d * r
    e_mu = (n + 2) * U * mean(x.abs())
    e_d = e_mu + U * d.abs()
    rho = 0.5 * ((n + 3) * U * var + 2 * e_mu * mean(d.abs()) + e_mu ** 2) / (var + eps) + 5 * U
    e_x = r * e_d + xh.abs() * (rho + U)
    if gy is None:
        b = torch.zeros_like(w) if b is None else b.double()
        y = xh * w + b
        return {"y": y}, {"y": w.abs() * (r * e_d + xh.abs() * (rho + 3 * U)) + U * y.abs() + U * b.abs()}
    gy = gy.double()
    a = gy * w
    skip = torch.zeros_like(a) if skip is None else skip.double()
    ma, al = mean(a), mean(a * xh)
    inner = a - ma - xh * al
    e_al = (n + 4) * U * mean((a * xh).abs()) + mean(a.abs() * e_x)
    gx = r * inner + skip
    e_gx = r * (U * a.abs() + (n + 2) * U * mean(a.abs()) + xh.abs() * e_al + al.abs() * e_x + 4 * U * (a.abs() + ma.abs() + (xh * al).abs()))
    e_gx += rho * (r * inner).abs() + U * (gx.abs() + skip.abs())
    return ({"gx": gx, "gw": (gy * xh).sum(0), "gb": gy.sum(0)},
            {"gx": e_gx, "gw": (rows + 2) * U * (gy * xh).abs().sum(0) + (gy.abs() * e_x).sum(0), "gb": rows * U * gy.abs().sum(0)})


def phi(z):
    return torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def linear(x, w, b, act, residual):
    """({out, z}, bounds)."""
    x, w = x.double(), w.double()
    K = x.shape[1]
    b = torch.zeros(w.shape[0], dtype=torch.float64, device=x.device) if b is None else b.double()
    z = x @ w.t() + b
    e_z = 2 * (K + 2) * U * (x.abs() @ w.abs().t() + b.abs())
    val = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.ndtr(z)}[act]()
    res = torch.zeros_like(z) if residual is None else residual.double()
    return {"out": val + res, "z": z}, {"out": 1.13 * e_z + 12 * U * val.abs() + U * (val.abs() + res.abs()), "z": e_z}


def linear_grad(x, w, z, act, go, bf16):
    """({gx, gw, gb}, bounds) with g = go act'(z)."""
    x, w, go = x.double(), w.double(), go.double()
    rows, N = go.shape
    if act == "none":
        g, e_g = go, torch.zeros_like(go)
    else:
        z = z.double()
        cdf, tail = torch.special.ndtr(z), z * phi(z)
        slope = cdf + tail if act == "gelu" else (z > 0).double()
        e_s = 8 * U * cdf + (z * z + 8) * U * tail.abs() if act == "gelu" else torch.zeros_like(z)
        g = go * slope
        e_g = go.abs() * e_s + U * g.abs()
    e_op = e_g + (H8 * g.abs() if bf16 and act != "none" else 0)
    return ({"gx": g @ w, "gw": g.t() @ x, "gb": g.sum(0)},
            {"gx": e_op @ w.abs() + 2 * (N + 2) * U * (g.abs() @ w.abs()), "gw": e_op.t() @ x.abs() + 2 * (rows + 2) * U * (g.abs().t() @ x.abs()),
             "gb": e_g.sum(0) + 2 * (rows + 2) * U * g.abs().sum(0)})


def check(name, got, val, far):
    """got within its bound, with half a step of its own type."""
    bound = far[name] + FLOOR + (H8 if got.dtype == torch.bfloat16 else U) * val[name].abs()
    err = (got.double() - val[name]).abs()
    assert torch.isfinite(got).all(), name
    worst = (err / bound).max().item() if err.numel() else 0.0
    assert worst <= 1.0, (name, worst)
    return worst
