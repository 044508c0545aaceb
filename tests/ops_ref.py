"""Float64 references of the stand-alone operators, on the CPU, with the bounds
their results may be off by.

u is half a step of fp32 (2^-24), h half a step of the output type (2^-8 for bf16,
2^-24 for fp32), both relative to the value."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
MAGS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def norm_rope(x, gain, rope, rows, halves, eps):
    """(result, magnitude): x [tokens][heads][dim], rope [n][rot / 2][2], rows [tokens].

    The sum of dim squares is off by at most dim u, its root by half of that; the divide, root, the
    two products and the rotation's products and sum add 8 u at most.  All of it is relative to the
    magnitude |a cos| + |b sin|, so a result is off by at most magnitude (dim / 2 + 8) u and its
    rounding, magnitude h."""
    x = x.double().cpu()
    dim = x.shape[-1]
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    mag = y.abs()
    if rope is None:
        return y, mag
    t = rope.double().cpu()[rows][:, None]
    half = rope.shape[1]
    p = torch.arange(half)
    i, j = (p, p + half) if halves else (2 * p, 2 * p + 1)
    a, b, c, s = y[..., i], y[..., j], t[..., 0], t[..., 1]
    out = y.clone()
    out[..., i], out[..., j] = a * c - b * s, a * s + b * c
    mag[..., i], mag[..., j] = (a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()
    return out, mag


def norm_bound(mag, dim, dtype):
    return mag * ((dim / 2 + 8) * U + HALF[dtype]) + 1e-37


def quantise(x):
    """(codes [..., dim / 2], scale bytes [..., dim / 32]) as uint8."""
    g = x.double().cpu().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    finite = torch.isfinite(g).all(-1)
    top = torch.where(finite[..., None], g, torch.zeros_like(g)).abs().amax(-1)
    m, ex = torch.frexp(top)                        # top = m 2^ex, m in [0.5, 1)
    byte = (ex - 3 + (m >= 0.875) + 127).clamp_min(1)
    byte = torch.where(top == 0, torch.ones_like(byte), byte)
    y = (g / torch.pow(2.0, byte.double() - 127)[..., None]).abs()
    code = torch.zeros(y.shape, dtype=torch.int64)
    best = torch.full_like(y, math.inf)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):              # even codes first: they win ties
        d = (y - MAGS[c]).abs()
        code = torch.where(d < best, torch.full_like(code, c), code)
        best = torch.minimum(best, d)
    code = (code + 8 * torch.signbit(g)).reshape(*x.shape[:-1], x.shape[-1] // 2, 2)
    byte = torch.where(finite, byte, torch.full_like(byte, 255))
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), byte.to(torch.uint8)


def dequantise(codes, scales):
    codes, scales = codes.cpu().long(), scales.cpu().double()
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    v = torch.where(c >= 8, -MAGS[c & 7], MAGS[c & 7]).reshape(*scales.shape, 32)
    s = torch.where(scales == 255, torch.full_like(scales, math.nan), torch.pow(2.0, scales - 127))
    return (v * s[..., None]).flatten(-2)


def attention(q, k, v, scale, kv_of, kv_len, mask, weights_rounded):
    """(result, bound) of q [n_q][lq][hq][dim] over k, v [n_kv][lk][hkv][dim] (float64, CPU).

    With W = sum p |v| and A the largest scale * sum |q k|: a score is off by at most
    (dim + 8) u A, its weight by as much relative to itself, the two sums by (keys + 8) u, so
    a result by at most W (2 (dim + 8) u A + (2 keys + 16) u).  Weights rounded to bf16 (each
    off by at most 2^-8 of itself, and summed as rounded) add 2 * 2^-8 W; the result's own
    rounding is added by the caller's type."""
    n_q, lq, hq, dim = q.shape
    n_kv, lk, hkv, _ = k.shape
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros(q.shape, dtype=torch.float64)
    for i in range(n_q):
        j = int(kv_of[i]) if kv_of is not None else i
        if not 0 <= j < n_kv:
            continue
        n = lk if kv_len is None else min(max(int(kv_len[j]), 0), lk)
        left = torch.arange(n)
        if mask is not None:
            left = left[mask[j, :n].cpu() != 0]
        if left.numel() == 0:
            continue
        for h in range(hq):
            qq, kk, vv = q[i, :, h].double().cpu(), k[j, left, h * hkv // hq], v[j, left, h * hkv // hq]
            p = torch.softmax(scale * (qq @ kk.t()), -1)
            a = scale * (qq.abs() @ kk.abs().t()).amax(-1, keepdim=True)
            w = p @ vv.abs()
            out[i, :, h] = p @ vv
            bound[i, :, h] = w * (2 * (dim + 8) * U * a + (2 * left.numel() + 16) * U + (2.0 ** -7 if weights_rounded else 0))
    return out, bound + HALF[q.dtype] * (out.abs() + bound) + 1e-37


def rope_table(rows, rot, base=10000.0):
    half = rot // 2
    ang = torch.arange(rows, dtype=torch.float64)[:, None] * base ** (-torch.arange(half, dtype=torch.float64) / half)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()
