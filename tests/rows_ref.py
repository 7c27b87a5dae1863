"""Plain 64-bit forms of the layers on rows of values, with bounds on what 32-bit sums and the results' rounding may leave.

U32 = 2^-24 is half a step of fp32; half(t) that of the result's type.  A bound is (roundings in a row) x U32 x (sum of the
magnitudes added) + half(t) |result| + half of the type's smallest step, each line naming its roundings."""
import math

import torch

U32 = 2.0 ** -24
TYPES = (torch.float32, torch.bfloat16, torch.float16)


def half(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    f = torch.finfo(dtype)
    return f.tiny * f.eps / 2


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def act_slope(z, name):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), torch.ones_like(z))
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def product_bound(k, a):
    """A sum of k products with magnitudes summing to a.  Matrix instructions add 32 products at a time and may cut the sum
    off, a whole step 2 U32 of the running sum each time: k / 32 of them, and as many again for the products within the
    first; splitting fp32 operands leaves out 2 U32 of a product; the joins of a split k and the vector kernels' lane sums
    add at most 64 roundings."""
    return (2 * (k / 32 + 32) + 2 + 64) * U32 * a


def linear_fwd(x, w, bias, name, residual, dtype):
    """((out, bound), (pre, bound)) on the CPU in 64 bits."""
    x, w = x.double().cpu(), w.double().cpu()
    z, a = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z = z + bias.double().cpu()
        a = a + bias.double().cpu().abs()
    bz = product_bound(x.shape[1], a)
    y = act(z, name)
    # the steepest slopes are 1.13 (gelu) and 1.1 (silu); erfc, exp and the quotient are good to 16 U32 of the value, and of
    # z where the value is a small difference
    by = 1.2 * bz + (0 if name in ("none", "relu") else 1) * 16 * U32 * (y.abs() + z.abs() * 0.5)
    if residual is not None:
        r = residual.double().cpu()
        by = by + 2 * U32 * (y.abs() + r.abs())
        y = y + r
    return (y, by + half(dtype) * (y.abs() + by) + tiny(dtype)), (z, bz + half(dtype) * (z.abs() + bz) + tiny(dtype))


def linear_bwd(x, w, g, name, pre, dtype):
    """[(dx, bound), (dw, bound), (dbias, bound)]"""
    x, w, g = x.double().cpu(), w.double().cpu(), g.double().cpu()
    dz = g if pre is None else g * act_slope(pre.double().cpu(), name)
    # the slope: a sum of terms up to 0.5 |z| of 16 U32 each; then, for the products, dz in the operands' type
    err = torch.zeros_like(dz) if pre is None else g.abs() * 16 * U32 * (1 + pre.double().cpu().abs().clamp(max=16))
    held = err + (0 if dtype == torch.float32 or pre is None else half(dtype)) * dz.abs() + (tiny(dtype) if pre is not None else 0)
    big = dz.abs() + held
    out = []
    for r, e in ((dz @ w.t(), product_bound(dz.shape[1], big @ w.abs().t()) + held @ w.abs().t()),
                 (x.t() @ dz, product_bound(dz.shape[0], x.abs().t() @ big) + x.abs().t() @ held)):
        out.append((r, e + half(dtype) * (r.abs() + e) + tiny(dtype)))
    # a lane adds every 1024th row or more, 256 lanes' sums are joined, the rest is fp64
    b = dz.sum(0)
    e = (300 + dz.shape[0] / 256) * U32 * (dz.abs() + err).sum(0) + err.sum(0)
    out.append((b, e + half(dtype) * (b.abs() + e) + tiny(dtype)))
    return out


def layer_norm_fwd(x, gamma, beta, eps, dtype):
    """[(out, bound), (mean, bound), (rstd, bound)]"""
    x = x.double().cpu()
    c = x.shape[1]
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = (d * d).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    n = 64 + c / 1024  # 32 values a lane (more in rows past a workgroup's registers), 10 lane exchanges, 16 waves
    em = n * U32 * x.abs().mean(1, keepdim=True)
    # deviations: their own rounding and the mean's error, whose cross term cancels but for roundings; the root halves
    rel = 0.5 * ((n + 8) * U32 + (em * em + 2 * em * U32 * d.abs().amax(1, keepdim=True)) / (var + eps)) + 4 * U32
    y = d * rstd
    e = rstd * em + y.abs() * (rel + 4 * U32)
    if gamma is not None:
        y, e = y * gamma.double().cpu(), e * gamma.double().cpu().abs()
    if beta is not None:
        e = e + 2 * U32 * (y.abs() + beta.double().cpu().abs())
        y = y + beta.double().cpu()
    e = e + 2 * U32 * y.abs()
    return [(y, e + half(dtype) * (y.abs() + e) + tiny(dtype)), (mean[:, 0], em[:, 0] + tiny(torch.float32)),
            (rstd[:, 0], (rstd * rel)[:, 0])]


def layer_norm_bwd(x, g, gamma, mean, rstd, dtype):
    """[(dx, bound), (dgamma, bound), (dbeta, bound)] from the statistics as they are given"""
    x, g, mean, rstd = x.double().cpu(), g.double().cpu(), mean.double().cpu()[:, None], rstd.double().cpu()[:, None]
    rows, c = x.shape
    xh = (x - mean) * rstd
    ex = 3 * U32 * xh.abs()  # difference, product
    h = g if gamma is None else g * gamma.double().cpu()
    n = (64 + c / 1024) * U32
    m_h, m_hx = h.mean(1, keepdim=True), (h * xh).mean(1, keepdim=True)
    e_h = n * h.abs().mean(1, keepdim=True)
    e_hx = (n + 6 * U32) * (h * xh).abs().mean(1, keepdim=True)
    dx = rstd * (h - m_h - xh * m_hx)
    e = rstd * (8 * U32 * (h.abs() + m_h.abs() + (xh * m_hx).abs()) + e_h + xh.abs() * e_hx + ex * m_hx.abs())
    out = [(dx, e + half(dtype) * (dx.abs() + e) + tiny(dtype))]
    for r, a in (((g * xh).sum(0), (g * xh).abs().sum(0)), (g.sum(0), g.abs().sum(0))):
        e = (64 + rows / 128 + 8) * U32 * a  # rows a lane adds, lanes and waves, the products; the rest is fp64
        out.append((r, e + half(dtype) * (r.abs() + e) + tiny(dtype)))
    return out


def assert_within(got, want, what=""):
    value, bound = want
    got = got.double().cpu()
    assert got.shape == value.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(value)), f"{what}: NaN in other places"
    inf = torch.isinf(value)
    assert torch.equal(got[inf], value[inf]), f"{what}: infinities differ"
    ok = torch.isfinite(value)
    off = (got - value).abs()[ok] - bound.expand_as(value)[ok]
    if off.numel():
        i = int(off.argmax())
        assert float(off[i]) <= 0, f"{what}: {float(got[ok][i])!r} for {float(value[ok][i])!r}, bound {float(bound.expand_as(value)[ok][i]):.3g}"
