"""Plain 64-bit forms of the residual block's operators (norm, linear, gated pair) with the error that the kernels may have,
element by element.  An output may be off by half a step of its type relative to its value, and by what fp32 arithmetic on its
terms can lose: n 2^-24 times the sum of the terms' magnitudes for a sum of n products (every product and every addition rounds
once), 2^-20 relative for an activation or a statistic (16 roundings: exponential, division, a handful of products)."""
import math

import torch

F64 = torch.float64
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24
FN = 2.0 ** -20


def act(z, kind):
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    return torch.relu(z) if kind == "relu" else z


def act_grad(z, kind):
    if kind == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if kind == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return (z > 0).to(z.dtype) if kind == "relu" else torch.ones_like(z)


def product(a, b):
    """a b^T and its fp32 error"""
    ref = a.to(F64) @ b.to(F64).t()
    return ref, a.shape[1] * U * (a.to(F64).abs() @ b.to(F64).abs().t())


def within(name, got, ref, err):
    """got (any type) against ref (64 bits): |got - ref| <= err + half a step of got's type"""
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    lim = err + HALF[got.dtype] * (ref.abs() + err) + 1e-38
    d = (got.to(F64) - ref).abs()
    ok = (d <= lim) & torch.isfinite(got)
    assert bool(ok.all()), "%s: %d of %d off, worst %.3g times the bound" % (
        name, int((~ok).sum()), ok.numel(), float((d / lim).nan_to_num(float("inf")).max()))


def linear(x, w, bias, residual, kind):
    z, ez = product(x, w)
    if bias is not None:
        z = z + bias.to(F64)
        ez = ez + U * z.abs()
    y = act(z, kind)
    ey = 1.2 * ez + FN * z.abs() if kind != "none" else ez      # (the slopes are at most 1.13)
    if residual is not None:
        y = y + residual.to(F64)
        ey = ey + U * y.abs()
    return (z, ez), (y, ey)


def gated(x, wg, wu, bg, bu, kind):
    (a, ea), _ = linear(x, wg, bg, None, "none")
    (u, eu), _ = linear(x, wu, bu, None, "none")
    h = act(a, kind) * u
    eh = (1.2 * ea + FN * a.abs()) * (u.abs() + eu) + act(a, kind).abs() * eu + U * h.abs()
    return (a, ea), (u, eu), (h, eh)


def back(dz, ez, x, ws, dtype):
    """dx, dw and db with their errors from the gradients dz of the pre-activations (lists: one per matrix), which are rounded to
    the tensors' type before the products"""
    half = HALF[dtype]
    dx = edx = 0
    dws, dbs = [], []
    for d, e, w in zip(dz, ez, ws):
        r = e + half * (d.abs() + e)                            # how far the rounded dz is off
        n = d.shape[1] * U * len(dz)
        dx = dx + d @ w.to(F64)
        edx = edx + (r + n * (d.abs() + r)) @ w.to(F64).abs()
        dws.append((d.t() @ x.to(F64), (r + d.shape[0] * U * (d.abs() + r)).t() @ x.to(F64).abs()))
        dbs.append((d.sum(0), e.sum(0) + d.shape[0] * U * d.abs().sum(0)))
    return (dx, edx), dws, dbs


def norm(x, gamma, beta, layer, eps):
    xd = x.to(F64)
    D = x.shape[1]
    mean = xd.mean(-1, keepdim=True) if layer else torch.zeros_like(xd[:, :1])
    emean = D * U * xd.abs().mean(-1, keepdim=True) if layer else torch.zeros_like(mean)
    c = xd - mean
    ec = emean + U * c.abs()
    var = (c * c).mean(-1, keepdim=True)
    # relative error of 1 / sqrt(var + eps): half that of its argument
    evar = (D + 4) * U * var + (2 * c.abs() * ec).mean(-1, keepdim=True) * (0 if layer else 1) + emean * emean
    rstd = (var + eps) ** -0.5
    er = rstd * (0.5 * evar / (var + eps) + 4 * U)
    g = torch.ones(D, dtype=F64, device=x.device) if gamma is None else gamma.to(F64)
    y = c * rstd * g
    ey = (ec * rstd + c.abs() * er) * g.abs() + 4 * U * y.abs()
    if beta is not None and layer:
        y = y + beta.to(F64)
        ey = ey + U * y.abs()
    return (mean[:, 0], emean[:, 0]), (rstd[:, 0], er[:, 0]), (y, ey)


def norm_back(x, dy, rstd, mean, gamma, residual, layer):
    """from the statistics as given"""
    D = x.shape[1]
    r = rstd.to(F64)[:, None]
    c = x.to(F64) - (mean.to(F64)[:, None] if layer else 0)
    xh = c * r
    exh = 3 * U * xh.abs()
    g = dy.to(F64) * (1 if gamma is None else gamma.to(F64))
    s1, s2 = (g * xh).mean(-1, keepdim=True), g.mean(-1, keepdim=True) if layer else 0
    e1 = (D + 6) * U * (g * xh).abs().mean(-1, keepdim=True)
    e2 = (D + 2) * U * g.abs().mean(-1, keepdim=True) if layer else 0
    dx = (g - xh * s1 - s2) * r
    edx = (2 * U * g.abs() + exh * s1.abs() + xh.abs() * e1 + e2 + 3 * U * (g.abs() + (xh * s1).abs() + abs(s2))) * r
    if residual is not None:
        dx = dx + residual.to(F64)
        edx = edx + U * (dx.abs() + edx)
    M = x.shape[0]
    t = dy.to(F64) * xh
    return (dx, edx), (t.sum(0), (M + 4) * U * t.abs().sum(0)), (dy.to(F64).sum(0), M * U * dy.to(F64).abs().sum(0))
