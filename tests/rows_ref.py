"""Float64 references of layer norm, rows in 8 bits and their products, on the CPU, with the
bounds their results may be off by.

u is half a step of fp32 (2^-24), h half a step of the output type, relative to the value.  A sum
over a row is taken as at most 64 values in turn on a lane and then over lanes and waves in at
most 16 more additions: it is off by at most 80 u times the sum of magnitudes."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
SUM = 80 * U


def _table(p, groups, rows, dim, none):
    """Parameters [groups][dim] or None as [groups * rows][dim]."""
    if p is None:
        return torch.full((groups * rows, dim), none, dtype=torch.float64)
    return p.double().cpu().repeat_interleave(rows, 0)


def _gain(weight, groups, rows, dim, unit):
    w = _table(weight, groups, rows, dim, 0.0 if unit else 1.0)
    return w + 1.0 if unit else w


def layer_norm(x, weight, bias, groups, unit, eps):
    """(y, its bound without the output's rounding, mean, its bound, rstd, its relative bound).

    The mean is off by m = (SUM + 2 u) mean|x|, and by as much each centred value, which rounds by u
    of itself; their squares add up to the variance and m^2, off by SUM + 4 u relative; with eps, root
    and inverse rstd is off by SUM / 2 + 6 u + (m rstd)^2 relative.  A normalised value is off by rstd m
    and by that, the centring's and the product's rounding; gain (1 + weight rounds once) and bias add 2 u
    of the product and u of the result."""
    rows, dim = x.shape[0] // groups, x.shape[1]
    x = x.double().cpu()
    mean = x.mean(-1, keepdim=True)
    z = x - mean
    rstd = 1.0 / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
    gain, b = _gain(weight, groups, rows, dim, unit), _table(bias, groups, rows, dim, 0.0)
    n = z * rstd
    y = n * gain + b
    m = (SUM + 2 * U) * x.abs().mean(-1, keepdim=True)
    rel = SUM / 2 + 6 * U + (m * rstd) ** 2
    off = gain.abs() * (rstd * m + n.abs() * (rel + 4 * U)) + U * y.abs()
    return y, 1.01 * off + 1e-37, mean[:, 0], 1.01 * m[:, 0] + 1e-37, rstd[:, 0], 1.01 * rel[:, 0]


def layer_norm_grad(x, dy, weight, mean, rstd, groups, unit):
    """((dx, bound without its rounding), (dw, bound), (db, bound)) for the given statistics.

    n rounds twice, g = dy gain twice; their means are off by SUM + 6 u of the mean magnitudes (8 u for
    g n), and each of the four steps of dx by u of what it takes.  A sum over rows passes at most
    min(rows, 300) + 16 additions: a part's rows, the waves of a workgroup and the parts of a group."""
    rows, dim = x.shape[0] // groups, x.shape[1]
    x, dy = x.double().cpu(), dy.double().cpu()
    mean, rstd = mean.double().cpu()[:, None], rstd.double().cpu()[:, None]
    n = (x - mean) * rstd
    g = dy * _gain(weight, groups, rows, dim, unit)
    m1, m2 = g.mean(-1, keepdim=True), (g * n).mean(-1, keepdim=True)
    dx = rstd * (g - m1 - n * m2)
    off = rstd.abs() * (6 * U * g.abs() + (SUM + 10 * U) * g.abs().mean(-1, keepdim=True) +
                        n.abs() * (SUM + 14 * U) * (g * n).abs().mean(-1, keepdim=True)) + 2 * U * dx.abs()
    depth = (min(rows, 300) + 16) * U
    by = lambda t: t.reshape(groups, rows, dim).sum(1)
    return ((dx, 1.01 * off + 1e-37), (by(dy * n), 1.01 * (depth + 4 * U) * by((dy * n).abs()) + 1e-37),
            (by(dy), 1.01 * depth * by(dy.abs()) + 1e-37))


def to_codes(x):
    """(codes int8, scales fp32) of rows of x."""
    x = x.double().cpu()
    ok = torch.isfinite(x).all(-1)
    top = torch.where(ok[:, None], x, 0.0).abs().amax(-1)
    scale = (top / 127).float()
    s = scale.double()[:, None]
    q = torch.round(torch.where(ok[:, None], x, 0.0) / torch.where(s > 0, s, math.inf)).clamp(-127, 127)
    return q.to(torch.int8), torch.where(ok, scale, math.nan)


def matmul(codes, scales, wq, ws, bias, gelu):
    """(result, bound without the output's rounding) of codes [m][k] and wq [n][k].

    The sum is exact and rounds once on its way to fp32, once with the row's scale and once with the
    column's and the bias.  The GELU x / (1 + 2^z) has a slope of at most 1.13; z is off by 4 u of itself, so
    2^z by 3 |z| u and its own 2 u, and the sum, inverse and product add 4 u."""
    acc = codes.double().cpu() @ wq.double().cpu().t()
    p = acc * scales.double().cpu()[:, None] * ws.double().cpu()
    y = p + (0.0 if bias is None else bias.double().cpu())
    off = 2 * U * p.abs() + U * y.abs()
    if gelu:
        z = -2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3) / math.log(2.0)
        out = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
        # where 2^z leaves the range of fp32 the result is below 1e-36
        off = 1.13 * off + out.abs() * (3 * z.abs() + 8) * U
        y = out
    return y, 1.01 * off + 1e-35
