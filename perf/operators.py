"""Cases of the operators that stand by themselves: norms of queries and keys per head with their
rotation, cross attention to contexts of other and of ragged lengths, the 4-bit key/value cache
and the attention that reads it.

Each case is one pass through the public calls (``cs_qk_norm_rope``, ``cs_cross_attention``,
``cs_kv4_store`` with ``cs_kv4_load``, ``cs_kv4_attention``) or, with ``own`` false, the same
operator written with elementary torch operations in 32 bits.  Head layouts, token counts and text
lengths come from the workload registry (12 and 40 heads of 128, 4 of 64 and of 32; 297, 1,560 and
32,760 tokens; 19, 77 and 512 text tokens) and, for the shared-head and single-token forms, are
generic ones (32 query heads on 8, caches up to 131,072 rows).

The 4-bit cache holds e2m1 codes (magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6; the sign in bit 3), two to
a byte with the even channel in the low half, and one scale byte b = 2^(b - 127) per 32 channels:
codes [n_kv][heads][cap][dim / 2], scales [n_kv][heads][cap][dim / 32].
"""
import math
import random

import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------- cases
def _norm(name, **kw):
    return dict(name=name, kind="norm", **kw)


def _store(name, **kw):
    return dict(name=name, kind="store", **kw)


def _attn(name, **kw):
    return dict(name=name, kind="attn", **kw)


def listed():
    return [
        # The new token of eight sequences, 32 query heads on 8 key heads, at far positions:
        # nothing but latency.
        _norm("norm_tokens_gqa", tokens=8, hq=32, hk=8, dim=128, rot=128, halves=True, fp32=False, span=32768,
              head_gains=False),
        # Three latents of the ragged geometry in fp32, the type used to check bf16 results.
        _norm("norm_ragged_fp32", tokens=891, hq=4, hk=4, dim=64, rot=64, halves=False, fp32=True, span=0,
              head_gains=True),
        # q and k of one 480p video at 14B widths, as views of the fused projection's output.
        _norm("norm_video_40h", tokens=32760, hq=40, hk=40, dim=128, rot=128, halves=False, fp32=False, span=0,
              head_gains=True),
        # The new token of sixteen sequences goes into their caches.
        _store("store_tokens", tokens=16, n_kv=16, cap=4096, heads=8, dim=128, fp32=False),
        # Text keys and values of all 30 blocks for four prompts.
        _store("store_prompts", tokens=61440, n_kv=120, cap=512, heads=12, dim=128, fp32=False),
        # One token of eight sequences against an encoder's states, 0 to 8,192 of them.
        _attn("attn_token_gqa", n_q=8, n_kv=8, lq=1, lk=8192, hq=32, hkv=8, dim=128, fp32=False, spread=1.0,
              mask=False, kv4=False),
        # Two latents each of three prompts of the ragged geometry, with dropped tokens, fp32.
        _attn("attn_ragged_fp32", n_q=6, n_kv=3, lq=297, lk=77, hq=4, hkv=4, dim=64, fp32=True, spread=0.8,
              mask=True, kv4=False),
        # One-frame 480p previews: two seeds each of four prompts of their own lengths.
        _attn("attn_frame_prompts", n_q=8, n_kv=4, lq=1560, lk=512, hq=12, hkv=12, dim=128, fp32=False, spread=0.9,
              mask=False, kv4=False),
        # Eight 480p videos of two prompts, the headline search's batch.
        _attn("attn_video_n8", n_q=8, n_kv=2, lq=32760, lk=512, hq=12, hkv=12, dim=128, fp32=False, spread=0.25,
              mask=False, kv4=False),
        # One token of sixteen sequences over 4-bit caches of up to 32,768 rows.
        _attn("kv4_token_batch", n_q=16, n_kv=16, lq=1, lk=32768, hq=32, hkv=8, dim=128, fp32=False, spread=0.9,
              mask=False, kv4=True),
        # One token of one sequence over a long 4-bit cache.
        _attn("kv4_token_long", n_q=1, n_kv=1, lq=1, lk=131072, hq=32, hkv=8, dim=128, fp32=False, spread=0.0,
              mask=False, kv4=True),
        # Five-frame 480p latents of four prompts whose text keys and values are kept in 4 bits.
        _attn("kv4_frames_prompts", n_q=4, n_kv=4, lq=7800, lk=512, hq=12, hkv=12, dim=128, fp32=False, spread=0.7,
              mask=False, kv4=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng):
    hkv = rng.choice([1, 2, 4, 8, 12])
    return hkv * rng.choice([1, 1, 2, 3, 4, 8] if hkv < 8 else [1, 1, 2, 4]), hkv, rng.choice([32, 64, 128, 128])


def draw(rng):
    kind = rng.choice(["norm", "store", "attn_token", "attn_rows", "kv4_token", "kv4_rows", "attn_fp32"])
    hq, hkv, dim = _draw_heads(rng)
    if kind == "norm":
        halves = rng.random() < 0.5
        rot = rng.choice([dim, dim, dim // 2])
        return dict(kind="norm", tokens=_log_int(rng, 1, 32760), hq=hq, hk=hkv, dim=dim, rot=rot, halves=halves,
                    fp32=rng.random() < 0.3, span=rng.choice([0, 4096, 32768]), head_gains=rng.random() < 0.5)
    if kind == "store":
        n_kv, cap = _log_int(rng, 1, 64), _log_int(rng, 16, 4096)
        return dict(kind="store", tokens=min(_log_int(rng, 1, 61440), n_kv * cap), n_kv=n_kv, cap=cap, heads=hkv,
                    dim=dim, fp32=rng.random() < 0.3)
    kv4 = kind.startswith("kv4")
    mask = rng.random() < 0.25
    if kind.endswith("token"):
        lk = _log_int(rng, 1, 131072 if kv4 else 32768)
        n = max(1, min(_log_int(rng, 1, 32), 524288 // (lk * hkv)))
        return dict(kind="attn", n_q=n, n_kv=n, lq=rng.choice([1, 1, 1, 2, 5]), lk=lk, hq=hq, hkv=hkv, dim=dim,
                    fp32=rng.random() < 0.2, spread=rng.choice([0.0, 0.5, 1.0]), mask=mask, kv4=kv4)
    n_kv, each = rng.randint(1, 4), rng.randint(1, 2)
    fp32 = kind == "attn_fp32"
    return dict(kind="attn", n_q=n_kv * each, n_kv=n_kv, lq=_log_int(rng, 60, 2000 if fp32 else 16000),
                lk=_log_int(rng, 5, 700), hq=min(hq, 24), hkv=hkv, dim=dim, fp32=fp32, spread=rng.uniform(0.0, 1.0),
                mask=mask, kv4=kv4)


# ------------------------------------------------------------------ inputs
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000 + salt)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _dtype(case):
    return torch.float32 if case["fp32"] else torch.bfloat16


def _lens(case):
    """Lengths of the contexts before they are dealt out: from lk down to (1 - spread) lk."""
    n = case["n_kv"]
    return [round(case["lk"] * (1.0 - case["spread"] * i / max(1, n - 1))) for i in range(n)]


def _rope_table(rows, rot):
    """(cos, sin) of position times frequency, the angle formed in 64 bits."""
    half = rot // 2
    freq = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    ang = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * freq[None, :]
    return torch.stack([ang.cos(), ang.sin()], dim=-1).float().contiguous()


def _quantise(x):
    """Codes and scale bytes of rows x [..., dim] in the cache's format."""
    g = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    amax = g.abs().amax(-1)
    # the power of two that puts the largest magnitude into [3.5, 7)
    scale = ((amax.view(torch.int32) + 0x200000) >> 23) - 2
    scale = scale.clamp(1, 253)
    y = g.double() / (scale << 23).view(torch.float32).double()[..., None]
    a = y.abs()
    # halfway values go to the even code
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * torch.signbit(y)).reshape(*x.shape[:-1], x.shape[-1] // 2, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scale.to(torch.uint8)


def _dequantise(codes, scales, mags):
    """The values that codes and scale bytes stand for, in 32 bits; mags: the eight magnitudes."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    v = torch.where(c >= 8, -mags[c & 7], mags[c & 7])
    v = v.reshape(*scales.shape, 32) * (scales.int() << 23).view(torch.float32)[..., None]
    return v.flatten(-2)


def _prepare_norm(case, seed):
    g = _gen(seed, 1)
    t, hq, hk, dim = case["tokens"], case["hq"], case["hk"], case["dim"]
    # q and k are views of a fused q, k, v projection
    x = _randn(g, t, hq + 2 * hk, dim) * (0.5 + torch.rand(dim, generator=g, device="cuda"))
    x = x.to(_dtype(case))
    rows = case["span"] or t
    heads = (hq, hk) if case["head_gains"] else (1, 1)
    s = {"q": x[:, :hq], "k": x[:, hq:hq + hk], "rope": _rope_table(rows, case["rot"]),
         "q_gain": 1.0 + 0.1 * _randn(g, heads[0], dim), "k_gain": 1.0 + 0.1 * _randn(g, heads[1], dim), "pos": None,
         "q_out": torch.empty(t, hq, dim, dtype=x.dtype, device="cuda"),
         "k_out": torch.empty(t, hk, dim, dtype=x.dtype, device="cuda")}
    if case["span"]:
        s["pos"] = torch.randint(0, rows, (t,), generator=g, device="cuda", dtype=torch.int32)
    if own:
        from paper_2607_23159_amd import binding as B
        s["plan"] = B.qk_norm_desc(s["q"], s["k"], s["q_out"], s["k_out"], s["q_gain"], s["k_gain"], s["rope"],
                                   style=B.CS_ROPE_HALVES if case["halves"] else B.CS_ROPE_PAIRS, eps=EPS)
    return s


def _prepare_store(case, seed):
    g = _gen(seed, 2)
    t, n, cap, h, dim = (case[x] for x in ("tokens", "n_kv", "cap", "heads", "dim"))
    kv = [(_randn(g, t, h, dim) * (0.3 + torch.rand(h, dim, generator=g, device="cuda"))).to(_dtype(case))
          for _ in range(2)]
    cache = [torch.zeros(n, h, cap, w, dtype=torch.uint8, device="cuda") for w in (dim // 2, dim // 32) * 2]
    if t == n:   # the next row of every sequence
        slots = torch.arange(n, device="cuda") * cap + torch.randint(0, cap, (n,), generator=g, device="cuda")
    else:
        slots = torch.randperm(n * cap, generator=g, device="cuda")[:t].sort().values
    s = {"k": kv[0], "v": kv[1], "cache": cache, "slots": slots, "slots32": slots.int(),
         "k_back": torch.empty_like(kv[0]), "v_back": torch.empty_like(kv[1])}
    if own:
        from paper_2607_23159_amd import binding as B
        s["plan"] = B.Kv4Cache(*cache)
    return s


def _prepare_attn(case, seed):
    g = _gen(seed, 3)
    n_q, n_kv, lq, lk, hq, hkv, dim = (case[x] for x in ("n_q", "n_kv", "lq", "lk", "hq", "hkv", "dim"))
    t = _dtype(case)
    lens = _lens(case)
    deal = random.Random(seed)
    deal.shuffle(lens)
    of = [i % n_kv for i in range(n_q)]
    deal.shuffle(of)
    s = {"q": (1.5 * _randn(g, n_q, lq, hq, dim)).to(t), "scale": 1.0 / math.sqrt(dim),
         "kv_len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "kv_of": torch.tensor(of, dtype=torch.int32, device="cuda"), "kv_mask": None,
         "o": torch.empty(n_q, lq, hq, dim, dtype=t, device="cuda")}
    k = _randn(g, n_kv, lk, hkv, dim)
    # values have a mean per channel, as an encoder's do
    v = _randn(g, n_kv, lk, hkv, dim) + 0.5 * _randn(g, hkv, dim)
    if case["mask"]:
        s["kv_mask"] = (torch.rand(n_kv, lk, generator=g, device="cuda") < 0.875).to(torch.uint8)
    if case["kv4"]:
        s["cache"] = [x.transpose(1, 2).contiguous() for x in (*_quantise(k), *_quantise(v))]
    else:
        s["k"], s["v"] = k.to(t), v.to(t)
    if own:
        from paper_2607_23159_amd import binding as B
        if case["kv4"]:
            s["kv"] = B.Kv4Cache(*s["cache"])
            s["plan"] = B.kv4_attn_desc(s["q"], s["kv"], s["o"], scale=s["scale"])
            need = B.cs_kv4_attention_workspace(s["plan"])
        else:
            s["plan"] = B.attn_desc(s["q"], s["k"], s["v"], s["o"], scale=s["scale"])
            need = B.cs_cross_attention_workspace(s["plan"])
        s["work"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


def prepare(case, seed):
    make = {"norm": _prepare_norm, "store": _prepare_store, "attn": _prepare_attn}[case["kind"]]
    s = make(case, seed)
    s["case"] = case
    s["mags"] = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    return s


# -------------------------------------------------------------------- runs
def _plain_norm_one(x, gain, rope, pos, case):
    y = x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * gain
    t = (rope[pos.long()] if pos is not None else rope)[:, None]
    r, rest = y[..., :case["rot"]], y[..., case["rot"]:]
    if case["halves"]:
        a, b = r.chunk(2, dim=-1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
    c, d = a * t[..., 0] - b * t[..., 1], a * t[..., 1] + b * t[..., 0]
    r = torch.cat([c, d], -1) if case["halves"] else torch.stack([c, d], -1).flatten(-2)
    return torch.cat([r, rest], -1).to(x.dtype)


def _plain_store_one(x, codes, scales, slots, mags):
    """Writes the rows x into a cache and reads them back."""
    n, h, cap = codes.shape[:3]
    seq, row = slots // cap, slots % cap
    q, s = _quantise(x)
    codes[seq, :, row], scales[seq, :, row] = q, s
    return _dequantise(codes[seq, :, row], scales[seq, :, row], mags).to(x.dtype)


def _plain_attn(s):
    case = s["case"]
    hkv, group = case["hkv"], case["hq"] // case["hkv"]
    if case["kv4"]:
        k, v = (_dequantise(s["cache"][i], s["cache"][i + 1], s["mags"]) for i in (0, 2))
    else:
        k, v = (s[x].float().transpose(1, 2) for x in ("k", "v"))
    of = s["kv_of"].long()
    left = torch.arange(case["lk"], device="cuda")[None] < s["kv_len"][:, None]
    if s["kv_mask"] is not None:
        left = left & (s["kv_mask"] != 0)
    left = left[of][:, None, None, :]
    k, v = k[of].transpose(2, 3).contiguous(), v[of].contiguous()
    q = s["q"].float().reshape(case["n_q"], case["lq"], hkv, group, case["dim"]).permute(0, 2, 1, 3, 4)
    q = q.reshape(case["n_q"], hkv, case["lq"] * group, case["dim"])
    p = torch.matmul(q * s["scale"], k).masked_fill_(~left, -math.inf)
    p.sub_(p.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    o = o.reshape(case["n_q"], hkv, case["lq"], group, case["dim"]).permute(0, 2, 1, 3, 4)
    return o.reshape(s["q"].shape).to(s["q"].dtype)


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        from paper_2607_23159_amd import binding as B
        if kind == "norm":
            B.cs_qk_norm_rope(s["plan"], s["q"], s["k"], s["q_out"], s["k_out"], s["q_gain"], s["k_gain"], s["rope"],
                              s["pos"])
            return s["q_out"], s["k_out"]
        if kind == "store":
            B.cs_kv4_store(s["plan"], s["k"], s["v"], s["slots32"])
            B.cs_kv4_load(s["plan"], s["k_back"], s["v_back"], s["slots32"])
            return s["k_back"], s["v_back"]
        if s["case"]["kv4"]:
            B.cs_kv4_attention(s["plan"], s["q"], s["kv"], s["o"], kv_of=s["kv_of"], kv_len=s["kv_len"],
                               kv_mask=s["kv_mask"], work=s["work"])
        else:
            B.cs_cross_attention(s["plan"], s["q"], s["k"], s["v"], s["o"], kv_of=s["kv_of"], kv_len=s["kv_len"],
                                 kv_mask=s["kv_mask"], work=s["work"])
        return s["o"]
    if kind == "norm":
        return (_plain_norm_one(s["q"], s["q_gain"], s["rope"], s["pos"], s["case"]),
                _plain_norm_one(s["k"], s["k_gain"], s["rope"], s["pos"], s["case"]))
    if kind == "store":
        c = s["cache"]
        return (_plain_store_one(s["k"], c[0], c[1], s["slots"], s["mags"]),
                _plain_store_one(s["v"], c[2], c[3], s["slots"], s["mags"]))
    return _plain_attn(s)


def work(case):
    e = 4 if case["fp32"] else 2
    if case["kind"] == "norm":
        values = case["tokens"] * (case["hq"] + case["hk"]) * case["dim"]
        table = min(case["span"] or case["tokens"], case["tokens"]) * case["rot"] * 4
        return {"bytes": 2 * values * e + table, "flops": 7 * values}
    row4 = case["dim"] // 2 + case["dim"] // 32
    if case["kind"] == "store":
        rows = 2 * case["tokens"] * case["heads"]
        # the rows in, their codes and scales out and in again, the values out
        return {"bytes": rows * 2 * (case["dim"] * e + row4), "flops": rows * case["dim"] * 4}
    lens, each = _lens(case), case["n_q"] // case["n_kv"]
    row = row4 if case["kv4"] else case["dim"] * e
    io = 2 * case["n_q"] * case["lq"] * case["hq"] * case["dim"] * e
    return {"bytes": io + sum(lens) * case["hkv"] * row * 2,
            "flops": 4 * case["lq"] * case["hq"] * case["dim"] * sum(lens) * each}


# ----------------------------------------------------------- 64-bit results
def _exact_norm_one(x, gain, table, rows, case):
    z = x.double()
    z = z / torch.sqrt(torch.einsum("thd,thd->th", z, z)[..., None] / z.shape[-1] + EPS) * gain.double()
    half = case["rot"] // 2
    p = torch.arange(half, device="cuda")
    i, j = (p, p + half) if case["halves"] else (2 * p, 2 * p + 1)
    w = torch.view_as_complex(table.double().contiguous())[rows][:, None, :]
    turned = torch.complex(z[..., i], z[..., j]) * w
    z = z.clone()
    z[..., i], z[..., j] = turned.real, turned.imag
    return z


def _values_of(cache):
    """Values [n][heads][rows][dim] of a pair of codes and scales, nibble by nibble, in 64 bits."""
    codes, scales = cache
    grid = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12, 0, -1, -2, -3, -4, -6, -8, -12], dtype=torch.float64, device="cuda") / 2
    v = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device="cuda")
    v[..., 0::2], v[..., 1::2] = grid[(codes % 16).long()], grid[(codes // 16).long()]
    return v * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, dim=-1)


def exact(case, seed):
    def on_grid(x):
        """x [rows][32] on the grid of its scale: the nearest of the signed magnitudes, by distance."""
        # even codes first: they win ties
        grid = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], dtype=torch.float64, device="cuda")
        top = x.abs().amax(-1, keepdim=True)
        m, ex = torch.frexp(top)               # top = m 2^ex, m in [0.5, 1)
        power = (ex - 3 + (m >= 0.875)).clamp_min(-126)
        unit = torch.ldexp(torch.ones_like(top), power)
        out = torch.empty_like(x)
        for b in range(0, x.shape[0], 1 << 20):
            y = x[b:b + (1 << 20)] / unit[b:b + (1 << 20)]
            best, kept = torch.full_like(y, math.inf), torch.zeros_like(y)
            for value in grid:
                d = (y.abs() - value).abs()
                kept = torch.where(d < best, value, kept)
                best = torch.minimum(d, best)
            out[b:b + (1 << 20)] = kept * torch.sign(y) * unit[b:b + (1 << 20)]
        return out

    s = prepare(case, seed)
    if case["kind"] == "norm":
        rows = s["pos"].long() if s["pos"] is not None else torch.arange(case["tokens"], device="cuda")
        return tuple(_exact_norm_one(s[x], s[x + "_gain"], s["rope"], rows, case) for x in ("q", "k"))
    if case["kind"] == "store":
        return tuple(on_grid(s[x].double().reshape(-1, 32)).reshape(s[x].shape) for x in ("k", "v"))
    group = case["hq"] // case["hkv"]
    if case["kv4"]:
        k, v = (_values_of(s["cache"][i:i + 2]) for i in (0, 2))
    else:
        k, v = (s[x].double().transpose(1, 2) for x in ("k", "v"))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for i, (j, n) in enumerate(zip(s["kv_of"].tolist(), s["kv_len"][s["kv_of"].long()].tolist())):
        at = torch.arange(n, device="cuda")
        if s["kv_mask"] is not None:
            at = at[s["kv_mask"][j, :n] != 0]
        if at.numel() == 0:
            continue
        for h in range(case["hq"]):
            w = (s["q"][i, :, h].double() @ k[j, h // group, at].t().contiguous()) * s["scale"]
            out[i, :, h] = torch.softmax(w, dim=-1) @ v[j, h // group, at]
    return out
