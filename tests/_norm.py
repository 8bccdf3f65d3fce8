"""float64 reference of the layer norm and its gradients, with bounds of the kernels' errors.

u = 2^-24 is fp32's largest relative rounding error. A row's sum is formed by threads that chain sixteen
values each (a 1024th of the row and a chunk where it is longer than they hold), a tree over a wave's 64 lanes and a chain
of at most 16 waves; a sum over rows by chains of a 256th of them, then at most 64 groups of a block, 16
partial sums of a part and 16 parts."""
import torch

U = 2.0 ** -24


def row_depth(C: int) -> float:
    return max(16.0, C / 1024 + 8) + 6 + 16


def column_depth(B: int, C: int) -> float:
    return (B / 256 + 1 if C <= 8192 else B) + 64 + 16 + 16


def norm_ref(x, weight, bias, eps):
    """(y, mean, rstd), their bounds before any rounding to a stored type, and what the backward reuses."""
    x = x.double()
    C = x.shape[-1]
    w = torch.ones(C, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    b = torch.zeros(C, dtype=torch.float64, device=x.device) if bias is None else bias.double()
    d = row_depth(C)
    mu = x.mean(-1, keepdim=True)
    e_mu = d * U * x.abs().mean(-1, keepdim=True) + 2 * U * mu.abs()
    v = x - mu
    e_v = e_mu + U * v.abs()
    var = v.square().mean(-1, keepdim=True)
    e_var = (2 * v.abs() * e_v + e_v.square()).mean(-1, keepdim=True) + (d + 3) * U * var
    s = (var + eps).rsqrt()
    # the sum with eps, root and quotient are rounded once each; eps itself is an fp32 number
    e_s = 1.1 * s * (0.5 * (e_var + U * (var + 2 * eps)) / (var + eps) + 4 * U)
    xh = v * s
    e_xh = e_v * s + v.abs() * e_s + e_v * e_s + U * xh.abs()
    y = xh * w + b
    e_y = w.abs() * e_xh + U * ((xh * w).abs() + b.abs()) + U * y.abs()
    return (y, mu[..., 0], s[..., 0]), (e_y, e_mu[..., 0], e_s[..., 0]), dict(w=w, s=s, xh=xh, e_s=e_s, e_xh=e_xh)


def norm_back_ref(ref, dy):
    """(dx, dweight, dbias) and their bounds."""
    w, s, xh, e_s, e_xh = (ref[k] for k in ("w", "s", "xh", "e_s", "e_xh"))
    dy = dy.double()
    C = dy.shape[-1]
    B = dy.numel() // C
    d, rows = row_depth(C), column_depth(B, C)
    g = dy * w
    m0, m1 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    e_m0 = (d + 1) * U * g.abs().mean(-1, keepdim=True) + 2 * U * m0.abs()
    e_m1 = (g.abs() * e_xh + (d + 2) * U * (g * xh).abs()).mean(-1, keepdim=True) + 2 * U * m1.abs()
    inner = g - m0 - xh * m1
    e_inner = e_m0 + xh.abs() * e_m1 + m1.abs() * e_xh + e_xh * e_m1 + 3 * U * (g.abs() + m0.abs() + (xh * m1).abs())
    dx = s * inner
    e_dx = s * e_inner + inner.abs() * e_s + e_inner * e_s + U * dx.abs()
    flat = lambda t: t.reshape(B, C)
    dw = flat(dy * xh).sum(0)
    e_dw = flat(dy.abs() * e_xh + (rows + 1) * U * (dy * xh).abs()).sum(0)
    db, e_db = flat(dy).sum(0), rows * U * flat(dy.abs()).sum(0)
    return (dx, dw, db), (e_dx, e_dw, e_db)
