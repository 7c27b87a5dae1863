"""Plain 64-bit forms of group norm with an activation, of dropout's mask and of 8-bit linear layers, with bounds on what
32-bit steps and the results' rounding may leave (U32 = 2^-24, half a step of fp32; half(t) that of the result's type)."""
import torch

from .rows_ref import U32, act, act_slope, assert_within, half, tiny  # noqa: F401

U64 = 2.0 ** -53


def bounds_of(offsets, rows, batch):
    """(first, end) of each sample, held to the array."""
    if offsets is None:
        return [(rows // batch * b, rows // batch * (b + 1)) for b in range(batch)]
    o = [min(max(int(v), 0), rows) for v in offsets]
    return [(o[b], max(o[b], o[b + 1])) for b in range(batch)]


def finish(z, e, name, dtype):
    """Value and bound of act(z) from z with error e: slopes are below 1.2; erfc, exp and the quotient are good to 16 U32 of the
    value, and of z where the value is a small difference; then the result's rounding."""
    y = act(z, name)
    e = 1.2 * e + (0 if name in ("none", "relu") else 1) * 16 * U32 * (y.abs() + z.abs() * 0.5)
    return y, e + half(dtype) * (y.abs() + e) + tiny(dtype)


def group_norm_fwd(x, groups, gamma, beta, samples, eps, name, dtype):
    """[(out of the samples' rows, bound), (mean, bound), (rstd, bound)] on the CPU, the rows in order"""
    x = x.double().cpu()
    c = x.shape[1]
    outs, means, rstds = [], [], []
    for first, end in samples:
        if first == end:
            means.append((torch.zeros(groups).double(), torch.zeros(groups).double()))
            rstds.append((torch.zeros(groups).double(), torch.zeros(groups).double()))
            continue
        v = x[first:end].view(end - first, groups, c // groups)
        n = (end - first) * (c // groups)
        mean = v.mean((0, 2))
        d = v - mean[:, None]
        var = (d * d).mean((0, 2))
        rstd = 1 / torch.sqrt(var + eps)
        # fp64 sums of up to n terms about the group's first value
        far = (v[0, :, 0] - mean).abs()
        em = (n + 8) * U64 * (v.abs().mean((0, 2)) + far)
        rel = 0.5 * ((n + 8) * U64 * (2 * var + 2 * far * far) + em * em) / (var + eps) + 2 * U64
        xh = d * rstd[:, None]
        # roundings: x - mean, what the mean's rounding leaves, rstd, its product with gamma
        e = 5 * U32 * xh.abs() + (em * rstd)[:, None] + U32 * U32 * (mean.abs() * rstd)[:, None] + xh.abs() * rel[:, None]
        z, e = xh.reshape(end - first, c), e.reshape(end - first, c)
        if gamma is not None:
            z, e = z * gamma.double().cpu(), e * gamma.double().cpu().abs()
        if beta is not None:
            z = z + beta.double().cpu()
        outs.append(finish(z, e + 2 * U32 * z.abs(), name, dtype))
        means.append((mean, em + U32 * mean.abs() + tiny(torch.float32)))
        rstds.append((rstd, rstd * (rel + 2 * U32)))
    out = tuple(torch.cat([o[i] for o in outs]) if outs else torch.zeros(0, c).double() for i in range(2))
    return [out] + [tuple(torch.stack([m[i] for m in s]) for i in range(2)) for s in (means, rstds)]


def group_norm_bwd(x, g, groups, gamma, beta, mean, rstd, samples, name, dtype):
    """[(dx of the samples' rows, bound), (dgamma, bound), (dbeta, bound)] from the statistics as they are given"""
    x, g, mean, rstd = x.double().cpu(), g.double().cpu(), mean.double().cpu(), rstd.double().cpu()
    c = x.shape[1]
    per = c // groups
    gam = torch.ones(c).double() if gamma is None else gamma.double().cpu()
    bet = torch.zeros(c).double() if beta is None else beta.double().cpu()
    # rows that one lane adds, and lanes of a workgroup whose sums are added in order: 128 or more vectors of four values or
    # more go side by side, up to 512 of eight
    side, most = max(1, 128 * 4 // c), max(1, 512 * 8 // c)
    outs, sums, errs = [], torch.zeros(2, c).double(), torch.zeros(2, c).double()
    for first, end in samples:
        if first == end:
            continue
        rows = end - first
        adds = (rows / side + 1 + most) * U32
        m, r = mean[samples.index((first, end))].repeat_interleave(per), rstd[samples.index((first, end))].repeat_interleave(per)
        xh = (x[first:end] - m) * r
        ex = 2 * U32 * xh.abs()
        z = xh * gam + bet
        slope = act_slope(z, name)
        es = torch.zeros_like(z)
        if name in ("gelu", "silu"):
            es = 1.2 * (ex * gam.abs() + U32 * z.abs()) + 16 * U32 * (1 + z.abs().clamp(max=16))
        dz = g[first:end] * slope
        ez = g[first:end].abs() * es + U32 * dz.abs()
        for k, (v, e) in enumerate(((dz * xh, ez * xh.abs() + dz.abs() * ex + U32 * (dz * xh).abs()), (dz, ez))):
            sums[k] += v.sum(0)
            errs[k] += e.sum(0) + adds * (v.abs() + e).sum(0)
        h, eh = dz * gam, ez * gam.abs() + U32 * (dz * gam).abs()

        def over(v):  # means over the sample's groups, back at every column
            return v.view(rows, groups, per).mean((0, 2)).repeat_interleave(per)

        m_h, m_hx = over(h), over(h * xh)
        e_h = over(eh) + (adds + 2 * U32) * over(h.abs())
        e_hx = over(eh * xh.abs() + h.abs() * ex) + (adds + 2 * U32) * over((h * xh).abs())
        dx = r * (h - m_h - xh * m_hx)
        e = r * (eh + e_h + xh.abs() * e_hx + ex * m_hx.abs() + 4 * U32 * (h.abs() + m_h.abs() + (xh * m_hx).abs()))
        outs.append((dx, e + half(dtype) * (dx.abs() + e) + tiny(dtype)))
    dx = tuple(torch.cat([o[i] for o in outs]) if outs else torch.zeros(0, c).double() for i in range(2))
    return [dx] + [(sums[k], errs[k] + half(dtype) * (sums[k].abs() + errs[k]) + tiny(dtype)) for k in range(2)]


def philox(counter, key):
    """The published generator, four 32-bit words in ten rounds, in Python's whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xffffffff, (p >> 32) ^ c[3] ^ k[1], p & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def words(first, count, seed, offset):
    """Random words of the values first .. first + count - 1."""
    out = []
    for block in range(first // 8, (first + count + 7) // 8):
        c = philox((block & 0xffffffff, block >> 32, offset & 0xffffffff, offset >> 32), (seed & 0xffffffff, seed >> 32))
        out += [(v >> s) & 0xffff for v in c for s in (0, 16)]
    return torch.tensor(out[first % 8:first % 8 + count])


def dropout(x, p, kept, residual, dtype):
    """(value, bound): the scale, the product and the sum are rounded to fp32."""
    t = round(p * 65536)
    y = torch.where(kept, x.double().cpu() * (65536 / (65536 - t) if t < 65536 else 0.0), torch.zeros(()).double())
    e = 2 * U32 * y.abs()
    if residual is not None:
        y = y + residual.double().cpu()
        e = e + U32 * (y.abs() + e)
    return y, e + half(dtype) * (y.abs() + e) + tiny(dtype)


def quantize(x):
    """(q, step) of rows, in fp32 steps as they are defined: exact."""
    x = x.float().cpu()
    most = x.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100)
    by = torch.full_like(most, 127.0)
    return torch.round(x * (by / most)).to(torch.int8), (most / by)[:, 0]


def linear_int8(q, step, w, w_step, bias, name, residual, dtype):
    """(out, bound): the exact sum to fp32, two products, the bias"""
    z = (q.double().cpu() @ w.double().cpu().t()) * step.double().cpu()[:, None] * w_step.double().cpu()
    e = 3 * U32 * z.abs() + tiny(torch.float32)
    if bias is not None:
        z = z + bias.double().cpu()
        e = e + U32 * (z.abs() + e)
    y, e = act(z, name), 1.2 * e + (0 if name in ("none", "relu") else 1) * 16 * U32 * (act(z, name).abs() + z.abs() * 0.5)
    if residual is not None:
        y = y + residual.double().cpu()
        e = e + U32 * (y.abs() + e)
    return y, e + half(dtype) * (y.abs() + e) + tiny(dtype)
