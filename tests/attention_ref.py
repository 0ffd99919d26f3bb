"""The window self-attention, its bias and AdamW in 64 bits on the CPU, as the formulas stand, with bounds for what the kernels may be off.

Bounds: u = 2^-24 (fp32) for every fp32 operation, h = 2^-8 (bf16, half a step) for every rounding to bf16, first order.
  s      (d + 3) u A with A the largest scale sum |q||k| + |bias|; the exponent's multiply-add, the base and 2^x: 4 u (largest |s|) + 8 u
  p      relative: r = that, and once more for the sum that divides it, and n u for the sum's own order
  out    (r + n u) sum p |v| ; bf16: + h sum p |v| (p as an operand) + h |out|
  D      n_d u sum |go out|; bf16: + sum |go| (h |out| + h sum p |v|), the saved out
  ds     p (r (|dp| + |D|) + d u sum |go v| + |error of D|); bf16 as an operand: + h |ds|
       and TINY (|dp| + |D|): powers below 2^-126 are flushed to zero
The gradients are sums of these against |k|, |q|, |go|, with n u for the order and h for the result in bf16.
"""
import math

import torch

U, H8, TINY = 2.0 ** -24, 2.0 ** -8, 2.0 ** -126   # TINY: a p below it is zero


def bucket_index(wh, ww, h, w, bucket):
    """Row of the table of every (query, key) of a window that holds h x w pixels; -1 where the bucket is none."""
    y, x = torch.arange(h).repeat_interleave(w), torch.arange(w).repeat(h)
    at = (y[:, None] - y[None] + wh - 1) * (2 * ww - 1) + (x[:, None] - x[None] + ww - 1)
    return at if bucket is None else bucket.reshape(-1).long()[at]


def bias_matrix(table, bucket, wh, ww, h=None, w=None):
    """[heads, N, N] in 64 bits."""
    at = bucket_index(wh, ww, h or wh, w or ww, bucket)
    ok = (at >= 0) & (at < table.shape[0])
    return torch.where(ok[..., None], table.double()[at.clamp(0, table.shape[0] - 1)], 0.0).permute(2, 0, 1)


def table_grad(g, n, at):
    """[n, heads] from g [heads, N, N]; entries of `at` outside the table take nothing."""
    ok = ((at >= 0) & (at < n)).reshape(-1)
    out = torch.zeros(n, g.shape[0], dtype=torch.float64)
    return out.index_add(0, at.reshape(-1)[ok], g.double().reshape(g.shape[0], -1).t()[ok].contiguous())


def attention(q, k, v, heads, wh, ww, table, bucket, scale, go=None, bf16=False):
    """(values, bounds): dicts with out, lse, and with `go` the gradients g_q, g_k, g_v, g_table.  q, k, v, go [B, H, W, heads * d] on the CPU."""
    q, k, v = q.double(), k.double(), v.double()
    B, H, W, C = q.shape
    d = C // heads
    val = {"out": torch.zeros_like(q), "lse": torch.zeros(B, heads, H, W, dtype=torch.float64)}
    if go is not None:
        go = go.double()
        val |= {n: torch.zeros_like(q) for n in ("g_q", "g_k", "g_v")}
        val["g_table"] = torch.zeros(table.shape[0], heads, dtype=torch.float64) if table is not None else None
    far = {n: None if x is None else torch.zeros_like(x) for n, x in val.items()}
    far["table_terms"] = torch.zeros_like(val["g_table"]) if val.get("g_table") is not None else None
    h8 = H8 if bf16 else 0.0
    for y in range(0, H, wh):
        for x in range(0, W, ww):
            h, w = min(wh, H - y), min(ww, W - x)
            n = h * w
            at = bucket_index(wh, ww, h, w, bucket)
            bias = bias_matrix(table, bucket, wh, ww, h, w) if table is not None else torch.zeros(heads, n, n, dtype=torch.float64)
            for b in range(B):
                part = (b, slice(y, y + h), slice(x, x + w))
                cut = lambda t: t[part].reshape(n, heads, d).transpose(0, 1)          # noqa: E731
                back = lambda t: t.transpose(0, 1).reshape(h, w, C)                    # noqa: E731
                qw, kw, vw = cut(q), cut(k), cut(v)
                s = scale * qw @ kw.transpose(1, 2) + bias
                lse = torch.logsumexp(s, 2, keepdim=True)
                p = torch.where(lse == -math.inf, 0.0, torch.exp(s - lse))
                out = p @ vw
                val["out"][part], val["lse"][b, :, y:y + h, x:x + w] = back(out), lse.reshape(heads, h, w)
                # bounds
                finite = torch.where(torch.isfinite(s), s.abs(), 0.0)
                A = (scale * qw.abs() @ kw.abs().transpose(1, 2) + torch.where(torch.isfinite(bias), bias.abs(), 0.0)).amax((1, 2), keepdim=True)
                r = 2 * U * ((d + 3) * A + 4 * finite.amax((1, 2), keepdim=True) + 8)
                mag = p @ vw.abs()
                far["out"][part] = back((r + 2 * n * U + h8) * mag + h8 * out.abs() + TINY * (1 + vw.abs().sum(1, keepdim=True)))
                far["lse"][b, :, y:y + h, x:x + w] = (r + n * U + 4 * U * torch.where(torch.isfinite(lse), lse.abs(), 0.0)).reshape(heads, h, w)
                if go is None:
                    continue
                gw = cut(go)
                dp, D = gw @ vw.transpose(1, 2), (gw * out).sum(2, keepdim=True)
                ds = p * (dp - D)
                val["g_q"][part], val["g_k"][part], val["g_v"][part] = back(scale * ds @ kw), back(scale * ds.transpose(1, 2) @ qw), back(p.transpose(1, 2) @ gw)
                e_out = (r + 2 * n * U + h8) * mag + h8 * out.abs()
                e_D = (gw.abs() * (e_out + (d + 1) * U * out.abs())).sum(2, keepdim=True)
                e_ds = p * ((r + n * U) * (dp.abs() + D.abs()) + (d + 2) * U * (gw.abs() @ vw.abs().transpose(1, 2)) + e_D) + 2 * U * ds.abs() + TINY * (dp.abs() + D.abs() + 1)
                op = e_ds + (h8 + 2 * n * U) * ds.abs()                               # as an operand of the products, with their order
                far["g_q"][part] = back(scale * op @ kw.abs() + (h8 + 2 * U) * (scale * ds @ kw).abs() + TINY)
                far["g_k"][part] = back(scale * op.transpose(1, 2) @ qw.abs() + (h8 + 2 * U) * (scale * ds.transpose(1, 2) @ qw).abs() + TINY)
                far["g_v"][part] = back((((r + 2 * n * U + h8) * p).transpose(1, 2)) @ gw.abs() + h8 * (p.transpose(1, 2) @ gw).abs() + TINY * (1 + gw.abs().sum(1, keepdim=True)))
                if table is not None:
                    t = table.shape[0]
                    val["g_table"] += table_grad(ds, t, at)
                    far["g_table"] += table_grad(e_ds, t, at)
                    far["table_terms"] += table_grad(ds.abs(), t, at)
    if go is not None and table is not None:
        # fp32 partial sums in a fixed order: at most one rounding per window and step of a lane, far fewer than 4096 of the terms' magnitudes
        far["g_table"] = far["g_table"] + 4096 * U * far["table_terms"] + h8 * val["g_table"].abs() + TINY
    far.pop("table_terms")
    return val, far


def check(got, ref, bound, what):
    got, ref = got.detach().double().cpu(), ref.double()
    same = torch.isfinite(got) == torch.isfinite(ref)
    assert same.all(), f"{what}: {int((~same).sum())} values finite on one side only"
    inf = ~torch.isfinite(ref)
    assert torch.equal(got[inf], ref[inf]) or torch.isnan(ref[inf]).any(), f"{what}: infinities differ"
    err = torch.where(inf, 0.0, (got - ref).abs())
    worst = (err / bound.clamp(min=1e-300)).max() if err.numel() else torch.zeros(())
    assert (err <= bound).all(), f"{what}: {int((err > bound).sum())} of {err.numel()} beyond the bound, worst {float(worst):.3g} of it, {float(err.max()):.3g}"
