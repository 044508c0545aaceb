"""Cases of the operators around projections in 8-bit integers: layer norm with its modulation,
forward and backward, rows to 8 bits and back, and the matrix product of 8-bit rows with 8-bit
weights.

Each case is one pass through the public calls (``cs_layer_norm``, ``cs_layer_norm_backward``,
``cs_i8_quantise`` with ``cs_i8_dequantise``, ``cs_matmul_i8``, or a norm to 8 bits with the product
that takes it) or, with ``own`` false, the same operator written with elementary torch operations.
Widths and token counts come from the workload registry (widths 256, 1536 and 5120, feed-forward
widths 512, 8960 and 13824; 297, 1,560 and 32,760 tokens a latent); the single-token forms are
generic.

Eight bits: a row (of activations) or an output channel (of weights) has one fp32 scale, its largest
magnitude over 127 rounded to fp32, and codes in -127..127, the integers nearest to value / scale,
halfway ones to the even one.
"""
import math

import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------- cases
def _norm(name, **kw):
    return dict(name=name, kind="norm", **kw)


def _grad(name, **kw):
    return dict(name=name, kind="grad", **kw)


def _rows8(name, **kw):
    return dict(name=name, kind="rows8", **kw)


def _mm(name, **kw):
    return dict(name=name, kind="mm", **kw)


def _proj(name, **kw):
    return dict(name=name, kind="proj", **kw)


def listed():
    return [
        # The new token of eight sequences at the largest width: nothing but latency.
        _norm("norm_tokens", groups=1, rows=8, dim=5120, x32=False, y32=False, mod=False, stats=False),
        # The residual stream of eight 480p videos in front of a projection, each with its own
        # modulation, and the statistics that a training step keeps.
        _norm("norm_videos", groups=8, rows=32760, dim=1536, x32=True, y32=False, mod=True, stats=True),
        # Three latents of the ragged geometry, fp32, a modulation each.
        _grad("grad_ragged_fp32", groups=3, rows=297, dim=256, x32=True, y32=True, mod=True),
        # One-frame 480p latents of eight seeds, fp32 residuals, a modulation each.
        _grad("grad_frames", groups=8, rows=1560, dim=1536, x32=True, y32=False, mod=True),
        # One 480p video at the largest width, one weight and bias for all of its tokens.
        _grad("grad_video", groups=1, rows=32760, dim=5120, x32=False, y32=False, mod=False),
        # The new token of sixteen sequences, to 8 bits and back.
        _rows8("rows8_tokens", rows=16, dim=5120, x32=False),
        # Feed-forward activations of a 480p video.
        _rows8("rows8_hidden", rows=32760, dim=8960, x32=False),
        # One token through the widest projection: the weights are all there is to read.
        _mm("mm_token", rows=1, n=13824, k=5120, act=False, o32=False),
        # Three latents of the ragged geometry through a small feed-forward up projection, fp32 out.
        _mm("mm_ragged", rows=891, n=512, k=256, act=True, o32=True),
        # One-frame 480p latents of eight seeds through the feed-forward down projection.
        _mm("mm_frames", rows=12480, n=1536, k=8960, act=False, o32=False),
        # One 480p video through the widest feed-forward up projection and its GELU.
        _mm("mm_video", rows=32760, n=13824, k=5120, act=True, o32=False),
        # One-frame 480p latent: modulated norm to 8 bits, then the query, key and value projection.
        _proj("proj_frame", groups=1, rows=1560, dim=1536, n=4608, x32=True, mod=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_dim(rng, hi):
    return rng.choice([256, 512, 1536, 5120, _log_int(rng, 16, hi), _log_int(rng, 16, hi)])


def draw(rng):
    kind = rng.choice(["norm", "grad", "rows8", "mm", "mm_few", "proj"])
    if kind in ("norm", "grad", "proj"):
        dim, groups = _draw_dim(rng, 8192), rng.choice([1, 1, 2, 3, 8])
        rows = min(_log_int(rng, 1, 32760), (1 << 27) // (dim * groups))
        case = dict(kind=kind, groups=groups, rows=max(1, rows), dim=dim, x32=rng.random() < 0.5,
                    mod=rng.random() < 0.5)
        if kind == "proj":
            case["rows"] = min(case["rows"], 8192 // groups)
            case["n"] = _log_int(rng, 64, 8192)
            return case
        case["y32"] = rng.random() < 0.3
        if kind == "norm":
            case["stats"] = rng.random() < 0.5
        return case
    if kind == "rows8":
        dim = _draw_dim(rng, 16384)
        return dict(kind=kind, rows=min(_log_int(rng, 1, 65536), (1 << 28) // dim), dim=dim, x32=rng.random() < 0.5)
    rows = _log_int(rng, 1, 64) if kind == "mm_few" else _log_int(rng, 65, 32760)
    n, k = _draw_dim(rng, 14000), _draw_dim(rng, 14000)
    return dict(kind="mm", rows=min(rows, 2_300_000_000_000 // (n * k)), n=n, k=k, act=rng.random() < 0.4,
                o32=rng.random() < 0.3)


# ------------------------------------------------------------------ inputs
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000 + salt)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _type(fp32):
    return torch.float32 if fp32 else torch.bfloat16


def _pad(n, to):
    return (n + to - 1) // to * to


def _buffer(rows, dim, dtype):
    """An uninitialised [rows][dim] tensor whose rows start on 16 bytes."""
    unit = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.empty(rows, _pad(dim, unit), dtype=dtype, device="cuda")[:, :dim]


def _residual_rows(gen, rows, dim, fp32):
    """Rows of a residual stream: channels of different spreads, a mean of their own."""
    x = _buffer(rows, dim, _type(fp32))
    scale = 0.5 + 2.0 * torch.rand(dim, generator=gen, device="cuda") ** 4
    shift = 0.5 * _randn(gen, dim)
    for i in range(0, rows, 32768):    # in slices: a residual stream is large
        n = min(32768, rows - i)
        x[i:i + n] = _randn(gen, n, dim) * scale + shift
    return x


def _to_codes(x):
    """(codes int8, scales fp32) of the rows of x, the quotients in 64 bits."""
    scale = (x.abs().amax(-1).double() / 127).float()
    q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    for i in range(0, x.shape[0], 8192):
        s = scale[i:i + 8192].double()[:, None]
        q[i:i + 8192] = torch.round(x[i:i + 8192].double() / torch.where(s > 0, s, 1.0)).to(torch.int8)
    return q, scale


def _weight(gen, n, k):
    return _to_codes(_randn(gen, n, k) * ((0.5 + torch.rand(n, 1, generator=gen, device="cuda")) / math.sqrt(k)))


def _modulation(gen, case, width):
    """Weight and bias per group, [groups][width] with rows on 16 bytes."""
    g = case["groups"]
    w, b = _buffer(g, width, torch.float32), _buffer(g, width, torch.float32)
    w.copy_(0.3 * _randn(gen, g, width) + (0.0 if case["mod"] else 1.0))
    b.copy_(0.3 * _randn(gen, g, width))
    return w, b


def _prepare_norm(case, seed):
    g = _gen(seed, 1)
    total, dim = case["groups"] * case["rows"], case["dim"]
    s = {"x": _residual_rows(g, total, dim, case["x32"])}
    s["w"], s["b"] = _modulation(g, case, dim)
    s["y"] = _buffer(total, dim, _type(case["y32"]))
    s["mean"], s["rstd"] = (torch.empty(total, device="cuda") if case["stats"] else None for _ in range(2))
    if own:
        from paper_2607_23159_amd import binding as B
        s["plan"] = B.layer_norm_desc(s["x"], s["y"], s["w"], s["b"], groups=case["groups"], unit_offset=case["mod"],
                                      eps=EPS)
    return s


def _prepare_grad(case, seed):
    g = _gen(seed, 2)
    groups, total, dim = case["groups"], case["groups"] * case["rows"], case["dim"]
    s = {"x": _residual_rows(g, total, dim, case["x32"]), "dy": _buffer(total, dim, _type(case["y32"]))}
    for i in range(0, total, 32768):
        n = min(32768, total - i)
        s["dy"][i:i + n] = _randn(g, n, dim)
    s["w"], s["b"] = _modulation(g, case, dim)
    s["mean"], s["rstd"] = torch.empty(total, device="cuda"), torch.empty(total, device="cuda")
    for i in range(0, total, 8192):    # what the forward pass kept
        x = s["x"][i:i + 8192].double()
        s["mean"][i:i + 8192] = x.mean(-1)
        s["rstd"][i:i + 8192] = torch.rsqrt(x.var(-1, unbiased=False) + EPS)
    s["dx"] = _buffer(total, dim, s["x"].dtype)
    s["dw"], s["db"] = _buffer(groups, dim, torch.float32), _buffer(groups, dim, torch.float32)
    if own:
        from paper_2607_23159_amd import binding as B
        s["plan"] = B.layer_norm_grad_desc(s["x"], s["dy"], s["w"], s["dx"], s["dw"], s["db"], groups=groups,
                                           unit_offset=case["mod"])
        need = B.cs_layer_norm_backward_workspace(s["plan"])
        s["work"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


def _prepare_rows8(case, seed):
    g = _gen(seed, 3)
    rows, dim = case["rows"], case["dim"]
    s = {"x": _residual_rows(g, rows, dim, case["x32"]), "codes": _buffer(rows, dim, torch.int8),
         "scales": torch.empty(rows, device="cuda"), "back": _buffer(rows, dim, _type(case["x32"]))}
    if own:
        from paper_2607_23159_amd import binding as B
        s["plan"] = B.i8_rows_desc(s["x"], s["codes"], s["scales"])
        s["plan_back"] = B.i8_rows_desc(s["back"], s["codes"], s["scales"])
    return s


def _product(s, case, gen, rows, k, out):
    """Weights in 8 bits, their layout, and the plan of a product of [rows][k] codes."""
    s["wq"], s["ws"] = _weight(gen, case["n"], k)
    s["bias"] = 0.1 * _randn(gen, case["n"])
    s["o"] = _buffer(rows, case["n"], out)
    if own:
        from paper_2607_23159_amd import binding as B
        s["weight"] = B.I8Weight(case["n"], k, device="cuda")
        wide = torch.zeros(case["n"], _pad(k, 16), dtype=torch.int8, device="cuda")
        wide[:, :k] = s["wq"]
        B.cs_i8_weight_pack(s["weight"], wide[:, :k], s["ws"])
        s["mm"] = B.matmul_i8_desc(s["codes"], s["scales"], s["weight"], s["o"],
                                   act=B.CS_ACT_GELU if case.get("act") else B.CS_ACT_NONE)
        need = B.cs_matmul_i8_workspace(s["mm"])
        s["work"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None


def _prepare_mm(case, seed):
    g = _gen(seed, 4)
    rows, k = case["rows"], case["k"]
    x = _residual_rows(g, rows, k, True)
    q, scale = _to_codes(x)
    s = {"codes": _buffer(rows, k, torch.int8), "scales": scale}
    s["codes"].copy_(q)
    _product(s, case, g, rows, k, _type(case["o32"]))
    return s


def _prepare_proj(case, seed):
    g = _gen(seed, 5)
    total, dim = case["groups"] * case["rows"], case["dim"]
    s = {"x": _residual_rows(g, total, dim, case["x32"]), "codes": _buffer(total, dim, torch.int8),
         "scales": torch.empty(total, device="cuda")}
    s["w"], s["b"] = _modulation(g, case, dim)
    _product(s, case, g, total, dim, torch.bfloat16)
    if own:
        from paper_2607_23159_amd import binding as B
        s["plan"] = B.layer_norm_desc(s["x"], s["codes"], s["w"], s["b"], groups=case["groups"],
                                      unit_offset=case["mod"], eps=EPS)
    return s


def prepare(case, seed):
    make = {"norm": _prepare_norm, "grad": _prepare_grad, "rows8": _prepare_rows8, "mm": _prepare_mm,
            "proj": _prepare_proj}[case["kind"]]
    s = make(case, seed)
    s["case"] = case
    return s


# -------------------------------------------------------------------- runs
def _gain(s):
    """Gains and biases [groups][1][dim]."""
    w = s["w"] + 1.0 if s["case"]["mod"] else s["w"]
    return w[:, None], s["b"][:, None]


def _plain_norm(s):
    """The normalised, modulated rows in 32 bits, with their mean and 1 / deviation."""
    c = s["case"]
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    gain, bias = _gain(s)
    y = (x * rstd).reshape(c["groups"], c["rows"], c["dim"]) * gain + bias
    return y.reshape(x.shape), mean[:, 0], rstd[:, 0]


def _plain_grad(s):
    c = s["case"]
    shape = (c["groups"], c["rows"], c["dim"])
    n = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    gain, _ = _gain(s)
    # sums over many rows, in 64 bits
    db = dy.reshape(shape).sum(1, dtype=torch.float64).float()
    dw = (dy * n).reshape(shape).sum(1, dtype=torch.float64).float()
    g = (dy.reshape(shape) * gain).reshape(n.shape)
    dx = (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True)) * s["rstd"][:, None]
    return dx.to(s["x"].dtype), dw, db


def _plain_mm(s, codes, scales):
    y = torch.matmul(codes.float(), s["wq"].float().t())
    y = y * scales[:, None] * s["ws"] + s["bias"]
    if s["case"].get("act"):
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    return y.to(s["o"].dtype)


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        from paper_2607_23159_amd import binding as B
        if kind == "norm":
            B.cs_layer_norm(s["plan"], s["x"], s["y"], s["w"], s["b"], mean=s["mean"], rstd=s["rstd"])
            return (s["y"], s["mean"], s["rstd"]) if s["case"]["stats"] else s["y"]
        if kind == "grad":
            B.cs_layer_norm_backward(s["plan"], s["x"], s["dy"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"],
                                     s["db"], work=s["work"])
            return s["dx"], s["dw"], s["db"]
        if kind == "rows8":
            B.cs_i8_quantise(s["plan"], s["x"], s["codes"], s["scales"])
            B.cs_i8_dequantise(s["plan_back"], s["codes"], s["scales"], s["back"])
            return s["back"], s["scales"]
        if kind == "proj":
            B.cs_layer_norm(s["plan"], s["x"], s["codes"], s["w"], s["b"], y_scale=s["scales"])
        B.cs_matmul_i8(s["mm"], s["codes"], s["scales"], s["weight"], s["o"], bias=s["bias"], work=s["work"])
        return s["o"]
    if kind == "norm":
        y, mean, rstd = _plain_norm(s)
        y = y.to(s["y"].dtype)
        return (y, mean, rstd) if s["case"]["stats"] else y
    if kind == "grad":
        return _plain_grad(s)
    if kind == "rows8":
        q, scale = _to_codes(s["x"])
        return (q.float() * scale[:, None]).to(s["x"].dtype), scale
    if kind == "proj":
        return _plain_mm(s, *_to_codes(_plain_norm(s)[0]))
    return _plain_mm(s, s["codes"], s["scales"])


def work(case):
    kind = case["kind"]
    ex = 4 if case.get("x32") else 2
    if kind in ("norm", "grad", "proj"):
        total, dim = case["groups"] * case["rows"], case["dim"]
        values, table = total * dim, 4 * case["groups"] * dim
        ey = 4 if case.get("y32") else 2
        if kind == "norm":
            return {"bytes": values * (ex + ey) + 2 * table + (8 * total if case["stats"] else 0), "flops": 8 * values}
        if kind == "grad":
            return {"bytes": values * (2 * ex + ey) + 3 * table + 8 * total, "flops": 14 * values}
        # the rows in, their codes out and in again, the weights, the outputs
        n = case["n"]
        return {"bytes": values * (ex + 2) + 2 * table + n * (dim + 8) + 2 * total * n,
                "flops": 8 * values + 2 * values * n}
    if kind == "rows8":
        values = case["rows"] * case["dim"]
        return {"bytes": values * (2 * ex + 2) + 8 * case["rows"], "flops": 6 * values}
    rows, n, k = case["rows"], case["n"], case["k"]
    return {"bytes": rows * k + n * k + rows * n * (4 if case["o32"] else 2) + 4 * rows + 8 * n, "flops": 2 * rows * n * k}


# ----------------------------------------------------------- 64-bit results
def _exact_norm_slice(x, w, b, mod):
    """Rows x of one group: (y, mean, 1 / deviation)."""
    z = x.double()
    var, mean = torch.var_mean(z, dim=-1, unbiased=False)
    dev = torch.sqrt(var + EPS)
    y = (z - mean[:, None]) / dev[:, None]
    return torch.addcmul(b.double() + (y if mod else 0.0), y, w.double()), mean, 1.0 / dev


def _exact_rows8(y):
    """(codes as doubles, scales) of rows in 64 bits; the format's scale is an fp32 number."""
    scale = (torch.maximum(y.amax(-1), -y.amin(-1)) / 127.0).float().double()
    t = y / torch.where(scale == 0.0, torch.ones_like(scale), scale)[:, None]
    low = torch.floor(t)
    odd = torch.remainder(low, 2.0)
    up = (t - low > 0.5) | ((t - low == 0.5) & (odd == 1.0))
    return low + up, scale


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    out = []
    if kind in ("norm", "proj"):
        for g in range(case["groups"]):
            for r in range(g * case["rows"], (g + 1) * case["rows"], 16384):
                x = s["x"][r:min(r + 16384, (g + 1) * case["rows"])]
                y, mean, rstd = _exact_norm_slice(x, s["w"][g], s["b"][g], case["mod"])
                if kind == "norm":
                    out.append((y, mean, rstd))
                else:
                    codes, scale = _exact_rows8(y)
                    out.append((codes @ s["wq"].double().t().contiguous() * scale[:, None] * s["ws"].double()
                                + s["bias"].double(),))
        parts = [torch.cat(p) for p in zip(*out)]
        return tuple(parts) if kind == "norm" and case["stats"] else parts[0]
    if kind == "grad":
        dx, dw, db = [], [], []
        for g in range(case["groups"]):
            at = slice(g * case["rows"], (g + 1) * case["rows"])
            gain = s["w"][g].double() + (1.0 if case["mod"] else 0.0)
            tw, tb = torch.zeros_like(gain), torch.zeros_like(gain)
            for r in range(at.start, at.stop, 8192):
                part = slice(r, min(r + 8192, at.stop))
                z, dy = s["x"][part].double(), s["dy"][part].double()
                var, mean = torch.var_mean(z, dim=-1, unbiased=False, keepdim=True)
                dev = torch.sqrt(var + EPS)
                n = (z - mean) / dev
                tb += torch.ones(1, dy.shape[0], dtype=torch.float64, device="cuda").matmul(dy)[0]
                tw += torch.linalg.vecdot(n, dy, dim=0)
                h = dy * gain
                along = torch.linalg.vecdot(h, n, dim=-1)[:, None] / case["dim"]
                dx.append((h - h.mean(-1, keepdim=True) - n * along) / dev)
            dw.append(tw)
            db.append(tb)
        return torch.cat(dx), torch.stack(dw), torch.stack(db)
    if kind == "rows8":
        parts = [_exact_rows8(s["x"][r:r + 8192].double()) for r in range(0, case["rows"], 8192)]
        return torch.cat([c * t[:, None] for c, t in parts]), torch.cat([t for _, t in parts])
    parts = []
    wide = s["wq"].double().t().contiguous()
    for r in range(0, case["rows"], 8192):
        y = s["codes"][r:r + 8192].double() @ wide
        y = torch.addcmul(s["bias"].double(), y * s["scales"][r:r + 8192].double()[:, None], s["ws"].double())
        parts.append(torch.nn.functional.gelu(y, approximate="tanh") if case["act"] else y)
    return torch.cat(parts)
