"""Plain 64-bit forms of the residual block in 8 bits, with the error that the kernels may have, element by element.

Quantisation of given values has none: a group's scale and codes are compared for equality.  A product of given codes has two errors.  The
matrix unit adds the products of eight neighbouring codes after dropping the bits that lie more than 13 below the leading bit of the
largest: seven products lose less than 2^-13 of it each.  Everything else is fp32: contraction length times 2^-24 of the sum
of the products' magnitudes.  Codes of values that a call itself computes may be those of any value within the value's own error."""
import torch

from tests.block_util import F64, FN, U, act, act_grad

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
DROP = 7 * 2.0 ** -13
# forward activations are those of the products in bf16: sigma to 2^-16 of its value, Phi to 2^-13 of it and 1.2e-7 < 2^-22 absolute
ACT = 2.0 ** -13 + 2.0 ** -22


def padded(x, rows, cols):
    R, C = x.shape
    full = torch.zeros((-(-R // rows) * rows, -(-C // cols) * cols), dtype=x.dtype, device=x.device)
    full[:R, :C] = x
    return full


def exponents(x, rows):
    """(blocks of rows, blocks of columns): the least e >= -127 with A <= 448 2^e, by trying powers of two in 64 bits"""
    x = x.to(F64)
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    a = padded(a, rows, 128)
    a = a.reshape(a.shape[0] // rows, rows, a.shape[1] // 128, 128).amax(dim=(1, 3))
    e = torch.floor(torch.log2(a.clamp_min(1e-300) / 448)).clamp_min(-128) - 1
    for _ in range(3):
        e = torch.where(a > 448 * torch.exp2(e), e + 1, e)
    return e.clamp_min(-127)


def spread(e, rows, shape):
    return e.repeat_interleave(rows, 0).repeat_interleave(128, 1)[:shape[0], :shape[1]]


def grid(v):
    """64-bit values of magnitude up to 448 (or not finite) on e4m3's grid, ties to even"""
    p = torch.frexp(v)[1].to(F64) - 1                       # |v| in [2^p, 2^(p+1))
    step = torch.exp2(p.clamp_min(-6) - 3)
    q = torch.round(v / step) * step
    return torch.where(torch.isfinite(v), q, torch.full_like(v, float("nan")))


def quant(x, rows=1):
    """codes as 64-bit values and scale bytes (blocks of columns, rows or blocks of rows)"""
    e = exponents(x, rows)
    return grid(x.to(F64) * torch.exp2(-spread(e, rows, x.shape))), (e + 127).to(torch.uint8).t().contiguous()


def requant(x, rows=1):
    """what the codes of x stand for"""
    e = exponents(x, rows)
    s = spread(e, rows, x.shape)
    return grid(x.to(F64) * torch.exp2(-s)) * torch.exp2(s)


def stands(q, scale):
    s = torch.exp2(scale.view(torch.uint8).to(F64) - 127).t()
    rows = 1 if s.shape[0] == q.shape[0] and (q.shape[0] > 1 or s.shape[0] == 1) else 128
    return q.to(F64) * spread(s, rows, q.shape)


def same_codes(q, scale, ref_q, ref_scale, name=""):
    assert q.dtype == E4M3 and scale.dtype == E8M0, (name, q.dtype, scale.dtype)
    assert q.shape == ref_q.shape and scale.shape == ref_scale.shape, (name, q.shape, scale.shape, ref_scale.shape)
    bad = scale.view(torch.uint8) != ref_scale
    assert not bool(bad.any()), "%s: %d of %d scales differ" % (name, int(bad.sum()), bad.numel())
    got = q.to(F64)
    bad = ~((got == ref_q) | (torch.isnan(got) & torch.isnan(ref_q)))
    assert not bool(bad.any()), "%s: %d of %d codes differ" % (name, int(bad.sum()), bad.numel())


def to_codes(x, rows=1):
    """codes and scales as the calls take them"""
    q, s = quant(x, rows)
    return q.to(torch.float32).to(E4M3).contiguous(), s.view(E8M0)


def product(a, b):
    """a b^T of two matrices of 64-bit values with its error"""
    a8, b8 = (padded(t, 1, 8) for t in (a, b))
    drop = torch.zeros((a.shape[0], b.shape[0]), dtype=F64, device=a.device)
    for k in range(0, a8.shape[1], 8):
        big = torch.zeros_like(drop)
        for j in range(k, k + 8):
            big = torch.maximum(big, a8[:, j, None].abs() * b8[None, :, j].abs())
        drop += big
    return a @ b.t(), DROP * drop + a.shape[1] * U * (a.abs() @ b.abs().t())


def linear(x, w, bias, residual, kind):
    """x, w: 64-bit values"""
    z, ez = product(x, w)
    if bias is not None:
        z = z + bias.to(F64)
        ez = ez + U * z.abs()
    y = act(z, kind)
    ey = 1.2 * ez + ACT * z.abs() if kind != "none" else ez
    if residual is not None:
        y = y + residual.to(F64)
        ey = ey + U * y.abs()
    return (z, ez), (y, ey)


def gated(x, wg, wu, bg, bu, kind):
    (a, ea), _ = linear(x, wg, bg, None, "none")
    (u, eu), _ = linear(x, wu, bu, None, "none")
    h = act(a, kind) * u
    eh = (1.2 * ea + (ACT if kind != "none" else 0) * a.abs()) * (u.abs() + eu) + act(a, kind).abs() * eu + 2 * U * h.abs()
    return (a, ea), (u, eu), (h, eh)


def coded(name, q, scale, v, ev):
    """codes and scales of values that are v but for ev"""
    e = scale.view(torch.uint8).to(F64).t() - 127
    lo, hi = exponents((v.abs() - ev).clamp_min(0), 1), exponents(v.abs() + ev, 1)
    assert e.shape == lo.shape, (name, e.shape, lo.shape)
    assert bool(((e >= lo) & (e <= hi)).all()), "%s: %d scales off" % (name, int(((e < lo) | (e > hi)).sum()))
    s = torch.exp2(spread(e, 1, v.shape))
    # within half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below its normal range) of a value within ev
    lim = ev + torch.maximum(2.0 ** -4 * (v.abs() + ev), 2.0 ** -10 * s)
    off = (q.to(F64) * s - v).abs()
    assert bool((off <= lim).all()), "%s: worst %.3g times the bound" % (name, float((off / lim).max()))


def requant_near(d, r):
    """Q(d) and how far Q of a value within r of d can be from it (r: 0 where d is exact)"""
    q = requant(d)
    lo, hi = requant(d - r), requant(d + r)
    # (a scale that changes moves every code of its group: the steps of the coarser one)
    e0, e1 = exponents((d.abs() - r).clamp_min(0), 1), exponents(d.abs() + r, 1)
    moved = torch.where(spread((e0 != e1).to(F64), 1, d.shape) > 0, 2.0 ** -4 * d.abs() + 2.0 ** -10 * torch.exp2(spread(e1, 1, d.shape)), torch.zeros_like(d))
    return q, torch.maximum((lo - q).abs(), (hi - q).abs()) + moved


def back(dz, ez, x, ws):
    """dx, dw and db with their errors.  dz: lists of gradients of pre-activations and their errors; ws: the weights (N, K) that codes stand for"""
    dx = edx = 0
    dws, dbs = [], []
    xt = requant(x.to(F64).t())
    for d, e, w in zip(dz, ez, ws):
        q, r = requant_near(d, e)
        p, ep = product(q, w.t())
        dx, edx = dx + p, edx + ep + r @ w.abs()
        q, r = requant_near(d.t().contiguous(), e.t().contiguous())
        p, ep = product(q, xt)
        dws.append((p, ep + r @ xt.abs().t()))
        dbs.append((d.sum(0), e.sum(0) + d.shape[0] * U * d.abs().sum(0)))
    return (dx, edx), dws, dbs


def gradients(kind, dy, z, u=None):
    """dz (or da and du) from the tensors as given, with their errors"""
    d, z = dy.to(F64), z.to(F64)
    if u is None:
        dz = d * act_grad(z, kind)
        return [dz], [torch.zeros_like(dz) if kind == "none" else FN * d.abs() * (1 + z.abs())]
    u = u.to(F64)
    return [d * u * act_grad(z, kind), d * act(z, kind)], [FN * (d * u).abs() * (1 + z.abs()), FN * (d * z).abs()]


def small_codes(gen, R, C, rows, device="cuda", spread_bits=3):
    """Codes whose products the matrix unit adds exactly: e4m3 values m 2^p, m = 1 ... 15/8, p = 0, 1, 2 (products from 2^0 to 2^6 in steps of
    2^-6), a third of them zero, and scales of a few neighbouring powers of two."""
    m = 1 + torch.randint(0, 8, (R, C), generator=gen, device=device).to(F64) / 8
    p = torch.randint(0, 3, (R, C), generator=gen, device=device).to(F64)
    sign = torch.randint(-1, 2, (R, C), generator=gen, device=device).to(F64)
    q = (sign * m * torch.exp2(p)).to(torch.float32).to(E4M3)
    s = torch.randint(127 - spread_bits, 127, (-(-C // 128), -(-R // rows)), generator=gen, device=device).to(torch.uint8)
    return q, s.view(E8M0)
