"""The stand-alone operators (per-head norms with rotation, cross attention to
ragged contexts, the 4-bit cache and its attention) against float64, at the sizes,
masks and layouts where they can go wrong."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import ops_ref as R
from paper_2607_23159_amd import binding as B

BF, FP = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def rnd(seed, *shape, dtype=FP, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype)


def guarded(shape, dtype, fill=-77.0):
    """A tensor inside a larger one of a known value, and a check that the rest still has it."""
    n = math.prod(shape)
    pad = 4096
    whole = torch.full((n + 2 * pad,), fill, dtype=dtype, device="cuda")
    t = whole[pad:pad + n].view(shape)

    def check():
        assert (whole[:pad] == fill).all() and (whole[pad + n:] == fill).all(), "written out of bounds"
    return t, check


def within(got, ref, bound, what):
    got = got.double().cpu()
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), "worst", float(((got - ref).abs() / bound).nan_to_num(9e9).max()),
                           "first", [int(x[0]) for x in bad.nonzero(as_tuple=True)])


# ----------------------------------------------------------- norm and rotation
NORM = [  # dtype, tokens, hq, hk, dim, rot, halves, head gains, positions
    (BF, 1, 1, 1, 128, 128, False, False, False),
    (BF, 1, 32, 8, 128, 128, True, False, True),
    (BF, 7, 12, 12, 128, 64, True, True, True),
    (BF, 297, 4, 4, 64, 64, False, True, False),
    (BF, 33, 5, 3, 96, 96, True, False, True),
    (BF, 5, 3, 1, 256, 128, False, True, True),
    (BF, 9, 2, 7, 16, 16, True, False, False),
    (BF, 66, 40, 40, 128, 0, False, True, False),
    (BF, 5000, 3, 2, 80, 32, False, False, True),
    (FP, 1, 4, 4, 32, 32, False, True, False),
    (FP, 297, 4, 4, 64, 64, False, True, False),
    (FP, 13, 9, 3, 112, 112, True, False, True),
    (FP, 3, 1, 1, 256, 256, True, True, True),
    (FP, 1000, 12, 12, 128, 96, False, False, False),
]


def _norm_case(dtype, t, hq, hk, dim, rot, head_gains, rows, seed=0):
    x = rnd(seed, t, hq + 2 * hk, dim, dtype=dtype).cuda()
    q, k = x[:, :hq], x[:, hq:hq + hk]
    qg = 1 + 0.2 * rnd(seed + 1, hq if head_gains else 1, dim).cuda()
    kg = 1 + 0.2 * rnd(seed + 2, hk if head_gains else 1, dim).cuda()
    rope = R.rope_table(rows, rot).cuda() if rot else None
    return q, k, qg, kg, rope


@pytest.mark.parametrize("dtype,t,hq,hk,dim,rot,halves,head_gains,with_pos", NORM)
def test_norm_rope(dtype, t, hq, hk, dim, rot, halves, head_gains, with_pos):
    rows = 50 if with_pos else max(1, t // 3)          # without positions the table repeats
    q, k, qg, kg, rope = _norm_case(dtype, t, hq, hk, dim, rot, head_gains, rows)
    pos = torch.randint(0, rows, (t,), generator=torch.Generator().manual_seed(5), dtype=torch.int32) if with_pos else None
    qo, check_q = guarded((t, hq, dim), dtype)
    ko, check_k = guarded((t, hk, dim), dtype)
    style = B.CS_ROPE_HALVES if halves else B.CS_ROPE_PAIRS
    d = B.qk_norm_desc(q, k, qo, ko, qg, kg, rope, style=style, eps=1e-5)
    B.cs_qk_norm_rope(d, q, k, qo, ko, qg, kg, rope, None if pos is None else pos.cuda())
    torch.cuda.synchronize()
    at = (pos.long() if pos is not None else torch.arange(t) % rows)
    for x, g, o, name in ((q, qg, qo, "q"), (k, kg, ko, "k")):
        ref, mag = R.norm_rope(x, g, rope, at, halves, 1e-5)
        within(o, ref, R.norm_bound(mag, dim, dtype), name)
    check_q()
    check_k()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_norm_skips_padding_and_marks_positions_past_the_table(dtype):
    t, hq, hk, dim, rows = 11, 6, 2, 64, 9
    q, k, qg, kg, rope = _norm_case(dtype, t, hq, hk, dim, 32, False, rows)
    pos = torch.tensor([0, 8, -1, 3, 9, -5, 2 ** 31 - 1, 1, -2 ** 31, 4, 8], dtype=torch.int32)
    qo = torch.full((t, hq, dim), 5.0, dtype=dtype, device="cuda")
    ko = torch.full((t, hk, dim), 5.0, dtype=dtype, device="cuda")
    d = B.qk_norm_desc(q, k, qo, ko, qg, kg, rope)
    B.cs_qk_norm_rope(d, q, k, qo, ko, qg, kg, rope, pos.cuda())
    for o, x, g in ((qo, q, qg), (ko, k, kg)):
        o = o.cpu()
        assert (o[pos < 0] == 5.0).all()
        assert torch.isnan(o[pos >= rows].float()).all()
        ok = (pos >= 0) & (pos < rows)
        ref, mag = R.norm_rope(x.cpu()[ok], g, rope, pos[ok].long(), False, 1e-6)
        within(o[ok], ref, R.norm_bound(mag, dim, dtype), "rows")


@pytest.mark.parametrize("dtype", [BF, FP])
def test_norm_in_place_one_side_and_zero_rows(dtype):
    q, k, qg, kg, rope = _norm_case(dtype, 40, 6, 6, 128, 128, True, 40)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    d = B.qk_norm_desc(q, k, qo, ko, qg, kg, rope)
    B.cs_qk_norm_rope(d, q, k, qo, ko, qg, kg, rope)
    # each side alone, in place, bitwise the same
    for x, o, g, a in ((q, qo, qg, "q"), (k, ko, kg, "k")):
        y = x.clone()
        args = (y, None, y, None, g, None) if a == "q" else (None, y, None, y, None, g)
        B.cs_qk_norm_rope(B.qk_norm_desc(*args, rope), *args, rope)
        assert torch.equal(y, o)
    # the strided view itself
    want = (qo.clone(), ko.clone())
    d = B.qk_norm_desc(q, k, q, k, qg, kg, rope)
    B.cs_qk_norm_rope(d, q, k, q, k, qg, kg, rope)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    # a row of zeros is divided by sqrt(eps) and stays zero
    z = torch.zeros(2, 1, 32, dtype=dtype, device="cuda")
    g = torch.ones(1, 32, device="cuda")
    B.cs_qk_norm_rope(B.qk_norm_desc(z, None, z, None, g, None), z, None, z, None, g, None)
    assert (z == 0).all()


@pytest.mark.parametrize("n", [1, 6, 300])
def test_norm_rows_do_not_depend_on_the_batch(n):
    q, k, qg, kg, rope = _norm_case(BF, 2000, 12, 4, 128, 128, True, 2000)
    outs = []
    for t in (2000, n):
        qo, ko = torch.empty(t, 12, 128, dtype=BF, device="cuda"), torch.empty(t, 4, 128, dtype=BF, device="cuda")
        d = B.qk_norm_desc(q[:t], k[:t], qo, ko, qg, kg, rope)
        B.cs_qk_norm_rope(d, q[:t], k[:t], qo, ko, qg, kg, rope)
        outs.append((qo[:n], ko[:n]))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


# --------------------------------------------------------------- 4-bit cache
def _cache(n, h, cap, dim, fill=0):
    return B.Kv4Cache(*(torch.full((n, h, cap, w), fill, dtype=torch.uint8, device="cuda")
                        for w in (dim // 2, dim // 32) * 2))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n,h,cap,dim,rows", [(1, 1, 1, 32, 1), (2, 3, 17, 64, 20), (3, 8, 40, 128, 77),
                                              (1, 12, 700, 128, 513), (5, 2, 33, 32, 101)])
def test_store_and_load(dtype, n, h, cap, dim, rows):
    x = rnd(3, rows, 2 * h, dim, dtype=dtype)
    x *= torch.exp2(torch.randint(-30, 30, (rows, 2 * h, dim // 32), generator=torch.Generator().manual_seed(1))
                    .float()).repeat_interleave(32, -1).to(dtype)     # scales far apart
    x[0, 0, :32] = 0
    x = x.cuda()
    k, v = x[:, :h], x[:, h:]
    g = torch.Generator().manual_seed(2)
    slots = torch.randperm(n * cap, generator=g)[:rows].int()
    slots[rows // 2] = -1 if rows > 1 else slots[0]
    if rows > 3:
        slots[1], slots[2] = n * cap, -2 ** 31
    cache = _cache(n, h, cap, dim, fill=0xA5)
    B.cs_kv4_store(cache, k, v, slots.cuda())
    want = [torch.full_like(t.cpu(), 0xA5) for t in cache.tensors]
    ok = (slots >= 0) & (slots < n * cap)
    seq, row = slots[ok].long() // cap, slots[ok].long() % cap
    for i, side in ((0, k), (2, v)):
        c, s = R.quantise(side[ok.cuda()])
        want[i][seq, :, row], want[i + 1][seq, :, row] = c, s
    for got, ref in zip(cache.tensors, want):
        assert torch.equal(got.cpu(), ref)
    ko = torch.full((rows, h, dim), 9.0, dtype=dtype, device="cuda")
    vo = torch.full((rows, h, dim), 9.0, dtype=dtype, device="cuda")
    B.cs_kv4_load(cache, ko, vo, slots.cuda())
    for o, side in ((ko, k), (vo, v)):
        assert (o.cpu()[~ok] == 9.0).all()
        assert torch.equal(o.cpu()[ok].double(), R.dequantise(*R.quantise(side[ok.cuda()])))


def test_store_rounds_every_bf16_value_and_marks_what_is_not_finite():
    # all finite bf16 values against a 6 in the same group, and groups that hold inf or NaN
    bits = torch.arange(65536, dtype=torch.int32)
    vals = (bits << 16).view(torch.float32)
    vals = vals[torch.isfinite(vals)]
    for top in (4.0, 6.5, 6.9921875, 2.0 ** -120, 2.0 ** 100):
        x = vals[vals.abs() <= top]
        x = torch.cat([x, torch.zeros(-x.numel() % 31)]).reshape(-1, 31)
        x = torch.cat([x, torch.full((x.shape[0], 1), top)], 1).reshape(-1, 1, 32).to(BF)
        for t in (BF, FP):
            k = x.to(t).cuda()
            cache = _cache(1, 1, k.shape[0], 32)
            B.cs_kv4_store(cache, k, -k)
            for i, y in ((0, k), (2, -k)):
                c, s = R.quantise(y)
                assert torch.equal(cache.tensors[i][0, 0].cpu(), c[:, 0]) and torch.equal(cache.tensors[i + 1][0, 0].cpu(), s[:, 0])
    x = torch.ones(4, 1, 64, dtype=FP)
    x[0, 0, 3], x[1, 0, 40], x[2, 0, 63] = math.inf, math.nan, -math.inf
    for t in (BF, FP):
        cache = _cache(1, 1, 4, 64)
        k = x.to(t).cuda()
        B.cs_kv4_store(cache, k, k)
        ko, vo = torch.empty_like(k), torch.empty_like(k)
        B.cs_kv4_load(cache, ko, vo)
        bad = ~torch.isfinite(x.reshape(4, 2, 32)).all(-1, keepdim=True).expand(4, 2, 32).reshape(4, 1, 64)
        assert torch.isnan(ko.cpu().float())[bad].all() and (ko.cpu().float()[~bad] == 1).all()
        assert torch.equal(torch.isnan(vo), torch.isnan(ko))


# ------------------------------------------------------------------ attention
ATTN = [  # dtype, n_q, n_kv, lq, lk, hq, hkv, dim, lengths, mask
    (BF, 1, 1, 1, 1, 1, 1, 128, "full", "none"),
    (BF, 2, 2, 1, 37, 4, 2, 64, "ragged", "none"),
    (BF, 3, 2, 5, 65, 8, 1, 32, "ragged", "holes"),
    (BF, 4, 3, 1, 700, 32, 8, 128, "ragged", "none"),
    (BF, 2, 1, 3, 2500, 6, 2, 128, "full", "holes"),
    (BF, 2, 3, 297, 19, 4, 4, 64, "ragged", "holes"),
    (BF, 2, 2, 100, 512, 12, 12, 128, "ragged", "none"),
    (BF, 1, 1, 385, 130, 3, 1, 128, "full", "none"),
    (BF, 3, 3, 200, 200, 4, 4, 32, "ragged", "empty"),
    (BF, 5, 2, 33, 64, 2, 2, 64, "strange", "holes"),
    (BF, 6, 4, 3000, 40, 16, 16, 32, "ragged", "none"),
    (BF, 7, 4, 2500, 70, 12, 12, 64, "ragged", "none"),
    (BF, 3, 2, 900, 330, 12, 12, 128, "ragged", "holes"),
    (BF, 2, 2, 200, 1500, 8, 4, 128, "ragged", "none"),
    (BF, 70, 3, 300, 60, 4, 4, 64, "ragged", "none"),
    (BF, 64, 5, 270, 90, 4, 4, 32, "strange", "holes"),
    (BF, 5, 3, 8, 2600, 16, 4, 128, "ragged", "none"),
    (BF, 3, 2, 21, 1100, 3, 1, 64, "ragged", "holes"),
    (BF, 2, 2, 64, 1030, 3, 1, 32, "strange", "none"),
    (BF, 2, 2, 193, 1030, 2, 2, 32, "ragged", "empty"),
    (FP, 1, 1, 1, 1, 1, 1, 32, "full", "none"),
    (FP, 3, 3, 1, 300, 8, 2, 128, "ragged", "holes"),
    (FP, 2, 2, 297, 77, 4, 4, 64, "ragged", "holes"),
    (FP, 2, 1, 50, 33, 6, 3, 32, "full", "none"),
    (FP, 2, 2, 65, 129, 4, 4, 128, "strange", "empty"),
    (FP, 1, 1, 2, 2500, 4, 1, 64, "full", "none"),
    (FP, 2, 1, 12, 60, 12, 4, 128, "ragged", "holes"),
    (FP, 1, 2, 40, 1100, 2, 2, 32, "ragged", "none"),
    (FP, 5, 3, 8, 2600, 16, 4, 128, "ragged", "none"),
    (FP, 2, 2, 1100, 150, 4, 4, 64, "ragged", "holes"),
    (FP, 3, 2, 1030, 77, 8, 8, 128, "ragged", "none"),
    (FP, 3, 2, 700, 300, 12, 12, 32, "strange", "empty"),
    (FP, 2, 2, 350, 60, 48, 12, 64, "ragged", "holes"),
    (FP, 1, 1, 1030, 4200, 8, 8, 32, "full", "holes"),
    (FP, 2, 2, 100, 1100, 96, 96, 32, "ragged", "none"),
]


def _lens(kind, n_kv, lk):
    if kind == "full":
        return None
    base = {"ragged": [lk, 0, 1, lk // 2, 3], "strange": [lk + 9, -4, 2 ** 31 - 1, lk // 3, -2 ** 31]}[kind]
    return torch.tensor((base * n_kv)[:n_kv], dtype=torch.int32)


def _masks(kind, n_kv, lk):
    if kind == "none":
        return None
    m = (torch.rand(n_kv, lk, generator=torch.Generator().manual_seed(8)) < 0.6).to(torch.uint8) * 255
    if kind == "empty":
        m[0] = 0
    return m


def _left(lens, mask, n_kv, lk):
    ok = torch.ones(n_kv, lk, dtype=torch.bool)
    if lens is not None:
        ok &= torch.arange(lk)[None] < lens[:, None].clamp(0, lk)
    if mask is not None:
        ok &= mask != 0
    return ok


def _of(n_q, n_kv, strange):
    of = [(3 * i + 1) % n_kv for i in range(n_q)]
    if strange:
        of[0], of[-1] = n_kv, -1
    return torch.tensor(of, dtype=torch.int32)


def _cuda(x):
    return None if x is None else x.cuda()


def _work(need):
    if not need:
        return None, lambda: None
    w, check = guarded((need,), torch.uint8, fill=201)
    w.random_(0, 256)       # whatever an earlier call left
    return w, check


@pytest.mark.parametrize("dtype,n_q,n_kv,lq,lk,hq,hkv,dim,lengths,masks", ATTN)
@pytest.mark.parametrize("layout", ["rows", "heads_first"])
def test_cross_attention(dtype, n_q, n_kv, lq, lk, hq, hkv, dim, lengths, masks, layout):
    lens, mask, of = _lens(lengths, n_kv, lk), _masks(masks, n_kv, lk), _of(n_q, n_kv, lengths == "strange")
    q = rnd(1, n_q, lq, hq, dim, dtype=dtype, scale=1.5)
    k, v = rnd(2, n_kv, lk, hkv, dim, dtype=dtype), rnd(3, n_kv, lk, hkv, dim, dtype=dtype) + 0.25
    left = _left(lens, mask, n_kv, lk)
    ref, bound = R.attention(q, k.double(), v.double(), 0.8 / math.sqrt(dim), of, lens, mask, dtype == BF)
    # what is left out may hold anything
    k[~left], v[~left] = math.nan, math.inf
    if layout == "rows":
        q, k, v = q.cuda(), k.cuda(), v.cuda()
    else:
        q, k, v = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (q, k, v))
    o, check = guarded((n_q, lq, hq, dim), dtype)
    d = B.attn_desc(q, k, v, o, scale=0.8 / math.sqrt(dim))
    w, check_w = _work(B.cs_cross_attention_workspace(d))
    B.cs_cross_attention(d, q, k, v, o, _cuda(of), _cuda(lens), _cuda(mask), w)
    torch.cuda.synchronize()
    within(o, ref, bound, "o")
    check()
    check_w()


@pytest.mark.parametrize("dtype,n_q,n_kv,lq,lk,hq,hkv,dim,lengths,masks", ATTN)
def test_kv4_attention(dtype, n_q, n_kv, lq, lk, hq, hkv, dim, lengths, masks):
    lens, mask, of = _lens(lengths, n_kv, lk), _masks(masks, n_kv, lk), _of(n_q, n_kv, lengths == "strange")
    q = rnd(1, n_q, lq, hq, dim, dtype=dtype, scale=1.5)
    parts = [R.quantise(rnd(s, n_kv, hkv, lk, dim) + 0.1 * s) for s in (2, 3)]
    k, v = (R.dequantise(*p).transpose(1, 2) for p in parts)
    ref, bound = R.attention(q, k, v, 1 / math.sqrt(dim), of, lens, mask, dtype == BF)
    out = (~_left(lens, mask, n_kv, lk))[:, None, :, None]
    cache = B.Kv4Cache(*(torch.where(out, torch.full_like(t, 255), t).cuda() for p in parts for t in p))
    q = q.cuda()
    o, check = guarded((n_q, lq, hq, dim), dtype)
    d = B.kv4_attn_desc(q, cache, o)
    w, check_w = _work(B.cs_kv4_attention_workspace(d))
    B.cs_kv4_attention(d, q, cache, o, _cuda(of), _cuda(lens), _cuda(mask), w)
    torch.cuda.synchronize()
    within(o, ref, bound, "o")
    check()
    check_w()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("lq", [1, 70])
def test_no_keys_give_zeros(dtype, kv4, lq):
    q = rnd(1, 2, lq, 4, 64, dtype=dtype).cuda()
    o = torch.full_like(q, 3.0)
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    if kv4:
        cache = _cache(2, 2, 50, 64, fill=255)
        d = B.kv4_attn_desc(q, cache, o)
        B.cs_kv4_attention(d, q, cache, o, kv_len=lens, work=_work(B.cs_kv4_attention_workspace(d))[0])
    else:
        k = torch.full((2, 50, 2, 64), math.nan, dtype=dtype, device="cuda")
        d = B.attn_desc(q, k, k, o)
        B.cs_cross_attention(d, q, k, k, o, kv_len=lens, work=_work(B.cs_cross_attention_workspace(d))[0])
        assert (o == 0).all()
        o.fill_(3.0)
        k = k[:, :0]       # room for no key at all
        d = B.attn_desc(q, k, k, o)
        B.cs_cross_attention(d, q, k, k, o, work=_work(B.cs_cross_attention_workspace(d))[0])
    assert (o == 0).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lq,lk,g", [(1, 3000, 4), (1, 90, 1), (3, 5000, 2), (40, 300, 3), (300, 200, 1)])
def test_scores_far_apart(dtype, lq, lk, g):
    """Scores up to the hundreds, the largest first, last and in the middle: weights underflow, the
    running maximum moves in every tile or never."""
    dim, hkv = 64, 2
    q = rnd(1, 3, lq, hkv * g, dim, dtype=dtype)
    k, v = rnd(2, 3, lk, hkv, dim, dtype=dtype), rnd(3, 3, lk, hkv, dim, dtype=dtype)
    ramp = torch.linspace(0.02, 30, lk)[None, :, None, None]
    k = k * torch.cat([ramp, ramp.flip(1), 30 - (ramp - 15).abs()], 0)
    k = k.to(dtype)
    ref, bound = R.attention(q, k.double(), v.double(), 1 / math.sqrt(dim), None, None, None, dtype == BF)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    o = torch.empty_like(q)
    d = B.attn_desc(q, k, v, o)
    B.cs_cross_attention(d, q, k, v, o, work=_work(B.cs_cross_attention_workspace(d))[0])
    within(o, ref, bound, "o")


def _ramps(n, lq, lk, hq, hkv, dim, dtype):
    """Scores up to the hundreds: the running maxima move in many tiles, in others for other queries."""
    q = rnd(1, n, lq, hq, dim, dtype=dtype)
    k, v = rnd(2, n, lk, hkv, dim, dtype=dtype), rnd(3, n, lk, hkv, dim, dtype=dtype)
    ramp = torch.linspace(0.02, 30, lk)[None, :, None, None]
    k = (k * torch.cat([ramp, ramp.flip(1), 30 - (ramp - 15).abs()], 0)[:n]).to(dtype)
    return q, k, v


def _attend(kv4, q, k, v, index=None, lens=None):
    """Attention of device tensors, k and v through a 4-bit cache if kv4."""
    o = torch.empty_like(q)
    if kv4:
        cache = _cache(k.shape[0], k.shape[2], k.shape[1], k.shape[3])
        B.cs_kv4_store(cache, k.flatten(0, 1), v.flatten(0, 1))
        d = B.kv4_attn_desc(q, cache, o)
        B.cs_kv4_attention(d, q, cache, o, index, lens, work=_work(B.cs_kv4_attention_workspace(d))[0])
    else:
        d = B.attn_desc(q, k, v, o)
        B.cs_cross_attention(d, q, k, v, o, index, lens, work=_work(B.cs_cross_attention_workspace(d))[0])
    return o


@pytest.mark.parametrize("dtype,kv4", [(BF, False), (BF, True), (FP, False), (FP, True)])
@pytest.mark.parametrize("lq,lk,dim", [(40, 1100, 64), (64, 1100, 128), (300, 1100, 64), (200, 1300, 32), (1130, 330, 64),
                                       (1060, 100, 128)])
def test_the_last_row_where_waves_lie_past_it(dtype, kv4, lq, lk, dim):
    """Rows that are no whole number of workgroups, in parts and over whole contexts: what a workgroup
    computes past the last row leaves that row as it is, alone and among other sets."""
    q, k, v = _ramps(3, lq, lk, 2, 2, dim, dtype)
    kk, vv = k.double(), v.double()
    if kv4:
        kk, vv = (R.dequantise(*R.quantise(x)) for x in (k, v))
    ref, bound = R.attention(q, kk, vv, 1 / math.sqrt(dim), None, None, None, dtype == BF)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    whole = _attend(kv4, q, k, v)
    within(whole, ref, bound, "o")
    for _ in range(3):
        for i in range(3):
            alone = _attend(kv4, q[i:i + 1], k, v, torch.tensor([i], dtype=torch.int32, device="cuda"))
            assert torch.equal(alone[0], whole[i]), i
        assert torch.equal(_attend(kv4, q, k, v), whole)


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lq,lk,hq,hkv,dim", [(1, 4000, 8, 2, 128), (5, 600, 12, 12, 64), (333, 512, 4, 4, 128),
                                              (1000, 77, 6, 3, 32), (1100, 600, 8, 8, 64)])
def test_attention_does_not_depend_on_the_batch(kv4, dtype, lq, lk, hq, hkv, dim):
    n = 6
    q = rnd(1, n, lq, hq, dim, dtype=dtype).cuda()
    lens = torch.tensor([lk, lk // 2, 1, lk - 1, 0, lk], dtype=torch.int32, device="cuda")
    of = torch.tensor([5, 3, 0, 1, 2, 4], dtype=torch.int32, device="cuda")
    k, v = rnd(2, n, lk, hkv, dim, dtype=dtype).cuda(), rnd(3, n, lk, hkv, dim, dtype=dtype).cuda()
    cache = _cache(n, hkv, lk, dim)
    B.cs_kv4_store(cache, k.flatten(0, 1), v.flatten(0, 1))

    def call(qq, index):
        o = torch.empty_like(qq)
        if kv4:
            d = B.kv4_attn_desc(qq, cache, o)
            B.cs_kv4_attention(d, qq, cache, o, index, lens, work=_work(B.cs_kv4_attention_workspace(d))[0])
        else:
            d = B.attn_desc(qq, k, v, o)
            B.cs_cross_attention(d, qq, k, v, o, index, lens, work=_work(B.cs_cross_attention_workspace(d))[0])
        return o

    whole = call(q, of)
    for i in range(n):
        assert torch.equal(call(q[i:i + 1], of[i:i + 1]), whole[i:i + 1]), i
    assert torch.equal(call(q, of), whole)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lq,lk,dim,masked", [(200, 90, 64, True), (300, 1100, 128, False), (1100, 70, 32, True)])
def test_fewer_sets_than_contexts(dtype, lq, lk, dim, masked):
    """Each set's context is unpacked into the workspace, whichever it is and if two sets share it."""
    n = 9
    lens = torch.tensor([lk, 3, lk - 1, 0, lk + 5, 17, lk // 2, 1, lk], dtype=torch.int32)
    mask = _masks("holes", n, lk) if masked else None
    q = rnd(1, 6, lq, 2, dim, dtype=dtype)
    parts = [R.quantise(rnd(s, n, 2, lk, dim) + 0.1 * s) for s in (2, 3)]
    k, v = (R.dequantise(*p).transpose(1, 2) for p in parts)
    of = torch.tensor([8, 2, 2, n, -1, 3], dtype=torch.int32)
    ref, bound = R.attention(q, k, v, 1 / math.sqrt(dim), of, lens, mask, dtype == BF)
    cache = B.Kv4Cache(*(t.cuda() for p in parts for t in p))
    q = q.cuda()
    for sets in (slice(0, 6), slice(1, 3), slice(5, 6)):
        o, check = guarded((sets.stop - sets.start, lq, 2, dim), dtype)
        d = B.kv4_attn_desc(q[sets], cache, o)
        w, check_w = _work(B.cs_kv4_attention_workspace(d))
        B.cs_kv4_attention(d, q[sets], cache, o, of[sets].cuda(), lens.cuda(), _cuda(mask), w)
        torch.cuda.synchronize()
        within(o, ref[sets], bound[sets], "o")
        check()
        check_w()
    # without an index the sets read the first contexts
    o, check = guarded((2, lq, 2, dim), dtype)
    d = B.kv4_attn_desc(q[:2], cache, o)
    B.cs_kv4_attention(d, q[:2], cache, o, None, lens.cuda(), _cuda(mask), _work(B.cs_kv4_attention_workspace(d))[0])
    ref, bound = R.attention(q[:2].cpu(), k, v, 1 / math.sqrt(dim), None, lens, mask, dtype == BF)
    within(o, ref, bound, "o")


@pytest.mark.parametrize("dtype,kv4", [(BF, False), (BF, True), (FP, False), (FP, True)])
@pytest.mark.parametrize("lq,hq,hkv,dim,lk", [(129, 8, 1, 128, 4200), (1061, 2, 2, 64, 2300), (350, 6, 2, 32, 5001)])
def test_many_rows_of_few_heads_over_long_contexts(dtype, kv4, lq, hq, hkv, dim, lk):
    n = 3
    lens = torch.tensor([lk - 7, 300, 0], dtype=torch.int32)
    mask = _masks("holes", n, lk)
    q = rnd(1, n, lq, hq, dim, dtype=dtype, scale=1.5)
    k, v = rnd(2, n, lk, hkv, dim, dtype=dtype), rnd(3, n, lk, hkv, dim, dtype=dtype)
    kk, vv = k.double(), v.double()
    if kv4:
        kk, vv = (R.dequantise(*R.quantise(x)) for x in (k, v))
    ref, bound = R.attention(q, kk, vv, 1 / math.sqrt(dim), None, lens, mask, dtype == BF)
    q, k, v, lens, mask = (x.cuda() for x in (q, k, v, lens, mask))
    cache = _cache(n, hkv, lk, dim)
    B.cs_kv4_store(cache, k.flatten(0, 1), v.flatten(0, 1))

    def call(qq, index):
        o, check = guarded(tuple(qq.shape), dtype)
        if kv4:
            d = B.kv4_attn_desc(qq, cache, o)
            w, check_w = _work(B.cs_kv4_attention_workspace(d))
            B.cs_kv4_attention(d, qq, cache, o, index, lens, mask, w)
        else:
            d = B.attn_desc(qq, k, v, o)
            w, check_w = _work(B.cs_cross_attention_workspace(d))
            B.cs_cross_attention(d, qq, k, v, o, index, lens, mask, w)
        torch.cuda.synchronize()
        check()
        check_w()
        return o

    whole = call(q, None)
    within(whole, ref, bound, "o")
    for i in range(n):
        assert torch.equal(call(q[i:i + 1], torch.tensor([i], dtype=torch.int32, device="cuda"))[0], whole[i])


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lq,lk,g", [(7, 1200, 4), (60, 300, 3), (400, 200, 1), (1100, 70, 8)])
def test_a_query_of_nans_leaves_the_others(kv4, dtype, lq, lk, g):
    q = rnd(1, 1, lq, 8, 64, dtype=dtype).cuda()
    k, v = rnd(2, 1, lk, 8 // g, 64, dtype=dtype).cuda(), rnd(3, 1, lk, 8 // g, 64, dtype=dtype).cuda()
    cache = _cache(1, 8 // g, lk, 64)
    B.cs_kv4_store(cache, k.flatten(0, 1), v.flatten(0, 1))

    def call(qq):
        o = torch.empty_like(qq)
        if kv4:
            d = B.kv4_attn_desc(qq, cache, o)
            B.cs_kv4_attention(d, qq, cache, o, work=_work(B.cs_kv4_attention_workspace(d))[0])
        else:
            d = B.attn_desc(qq, k, v, o)
            B.cs_cross_attention(d, qq, k, v, o, work=_work(B.cs_cross_attention_workspace(d))[0])
        return o

    whole = call(q)
    q[0, 3, 5] = math.nan
    got = call(q)
    assert got[0, 3, 5].isnan().all()
    got[0, 3, 5] = whole[0, 3, 5]
    assert torch.equal(got, whole)


@pytest.mark.parametrize("dtype,kv4", [(BF, False), (BF, True), (FP, False), (FP, True)])
@pytest.mark.parametrize("lq,lk,hq,hkv", [(7, 1200, 8, 2), (3, 400, 8, 2), (20, 300, 6, 2), (300, 200, 2, 2), (300, 1100, 2, 2),
                                          (1100, 330, 2, 2), (1100, 200, 8, 8)])
def test_a_query_does_not_depend_on_the_other_queries(dtype, kv4, lq, lk, hq, hkv):
    """Bitwise, where the others' running maxima move at other keys than its own."""
    q, k, v = _ramps(1, lq, lk, hq, hkv, 64, dtype)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    whole = _attend(kv4, q, k, v)
    keep = torch.arange(lq, device="cuda") % 3 == 1
    for scale in (0.0, 3.0):
        other = (scale * rnd(7, 1, lq, hq, 64)).to(dtype).cuda()
        other[:, keep] = q[:, keep]
        assert torch.equal(_attend(kv4, other, k, v)[:, keep], whole[:, keep]), scale


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lq,lk", [(1, 700), (40, 90), (1100, 130)])
def test_inputs_that_are_broadcast(dtype, lq, lk):
    """Strides of zero: one query set for all, keys of one head and one context for all."""
    q, k, v = rnd(1, 1, lq, 8, 64, dtype=dtype), rnd(2, 1, lk, 1, 64, dtype=dtype), rnd(3, 2, lk, 1, 64, dtype=dtype)
    lens = torch.tensor([lk, lk // 2 + 1], dtype=torch.int32)
    full = q.expand(3, -1, -1, -1), k.expand(2, -1, 8, -1), v.expand(-1, -1, 8, -1)
    of = _of(3, 2, False)
    ref, bound = R.attention(full[0], full[1].double(), full[2].double(), 0.125, of, lens, None, dtype == BF)
    q, k, v = q.cuda().expand(3, -1, -1, -1), k.cuda().expand(2, -1, 8, -1), v.cuda().expand(-1, -1, 8, -1)
    o, check = guarded((3, lq, 8, 64), dtype)
    d = B.attn_desc(q, k, v, o)
    B.cs_cross_attention(d, q, k, v, o, of.cuda(), lens.cuda(), work=_work(B.cs_cross_attention_workspace(d))[0])
    within(o, ref, bound, "o")
    check()


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lq,lk,g", [(2, 1100, 4), (60, 300, 1), (1100, 70, 1)])
def test_scores_of_a_billion(kv4, dtype, lq, lk, g):
    """Scores up to 10^9 leave averages of the values: a weight's exponent is off by at most 64
    (half a step of 2^30), the same for all keys of a maximum."""
    q = rnd(1, 1, lq, 8, 64, dtype=dtype).cuda()
    k, v = rnd(2, 1, lk, 8 // g, 64, dtype=dtype).cuda(), rnd(3, 1, lk, 8 // g, 64, dtype=dtype).cuda()
    cache = _cache(1, 8 // g, lk, 64)
    B.cs_kv4_store(cache, k.flatten(0, 1), v.flatten(0, 1))
    o = torch.empty_like(q)
    top = (q.double().abs().sum(-1).max() * 1.2 * k.abs().max()).item()   # a stored key is below 7 / 6 of the largest
    if kv4:
        d = B.kv4_attn_desc(q, cache, o, scale=1e9 / top)
        B.cs_kv4_attention(d, q, cache, o, work=_work(B.cs_kv4_attention_workspace(d))[0])
    else:
        d = B.attn_desc(q, k, v, o, scale=1e9 / top)
        B.cs_cross_attention(d, q, k, v, o, work=_work(B.cs_cross_attention_workspace(d))[0])
    assert o.isfinite().all()
    assert (o.abs().amax() <= (1.2 if kv4 else 1.01) * v.abs().amax()).item()
    assert (o.abs().amax(-1) > 0).all()


@pytest.mark.parametrize("lq,hq", [(1100, 8), (300, 2), (1, 4)])
@pytest.mark.parametrize("exponent", [-100, -103, -120])
def test_fp32_values_near_the_smallest_number(lq, hq, exponent):
    """Bf16 terms end at 2^-133, the smallest number of their type: values lose bits below 2^-103, by at
    most half of that number each, whatever the weights, which sum to one."""
    q, k, v = rnd(1, 1, lq, hq, 64), rnd(2, 1, 100, hq, 64), rnd(3, 1, 100, hq, 64)
    v *= 2.0 ** exponent / v.abs().clamp_min(1e-3)
    v *= 1 + 0.9 * rnd(4, 1, 100, hq, 64).abs().clamp_max(1)
    ref, bound = R.attention(q, k.double(), v.double(), 0.125, None, None, None, False)
    o = _attend(False, q.cuda(), k.cuda(), v.cuda())
    within(o, ref, bound - 1e-37 + 2.0 ** -134 + 2.0 ** -149, "o")


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lq", [1, 150])
def test_rows_more_than_two_gib_apart(dtype, lq):
    """Row offsets of a context pass 2^31 bytes."""
    lk, dim, step = 600, 128, (1 << 22) if dtype == BF else (1 << 21)
    big = torch.empty((lk - 1) * step + dim, dtype=dtype, device="cuda")
    k = big.as_strided((1, lk, 1, dim), (lk * step, step, dim, 1))
    k.copy_(rnd(2, 1, lk, 1, dim, dtype=dtype))
    v = rnd(3, 1, lk, 1, dim, dtype=dtype).cuda()
    q = rnd(1, 1, lq, 2, dim, dtype=dtype).cuda()
    for kk, vv in ((k, v), (v, k)):
        ref, bound = R.attention(q.cpu(), kk.double().cpu(), vv.double().cpu(), 1 / math.sqrt(dim), None, None, None, dtype == BF)
        o = torch.empty_like(q)
        d = B.attn_desc(q, kk, vv, o)
        B.cs_cross_attention(d, q, kk, vv, o, work=_work(B.cs_cross_attention_workspace(d))[0])
        within(o, ref, bound, "o")


@pytest.mark.parametrize("dtype,lq", [(BF, 1), (BF, 200), (FP, 3), (FP, 150)])
def test_cache_rows_past_four_gib(dtype, lq):
    """Heads of the cache lie 4 GiB apart; only the first rows of the contexts are in use."""
    n, h, cap, dim, used = 2, 2, 1 << 26, 128, torch.tensor([130, 77], dtype=torch.int32)
    cache = B.Kv4Cache(*(torch.empty(n, h, cap, w, dtype=torch.uint8, device="cuda") for w in (64, 4, 64, 4)))
    k, v = rnd(2, n * 130, h, dim, dtype=dtype), rnd(3, n * 130, h, dim, dtype=dtype)
    slots = torch.cat([torch.arange(130), cap + torch.arange(130)]).int()
    B.cs_kv4_store(cache, k.cuda(), v.cuda(), slots.cuda())
    kk, vv = torch.empty_like(k).cuda(), torch.empty_like(v).cuda()
    B.cs_kv4_load(cache, kk, vv, slots.cuda())
    kk, vv = kk.cpu(), vv.cpu()
    for x, y in ((k, kk), (v, vv)):
        want = R.dequantise(*R.quantise(x.transpose(0, 1)))
        assert torch.equal(y.transpose(0, 1).double(), want)
    q = rnd(1, n, lq, h, dim, dtype=dtype)
    ref, bound = R.attention(q, kk.double().view(n, 130, h, dim), vv.double().view(n, 130, h, dim), 1 / math.sqrt(dim), None,
                             used, None, dtype == BF)
    q = q.cuda()
    o = torch.empty_like(q)
    d = B.kv4_attn_desc(q, cache, o)
    work = torch.empty(max(1, B.cs_kv4_attention_workspace(d)), dtype=torch.uint8, device="cuda")
    B.cs_kv4_attention(d, q, cache, o, kv_len=used.cuda(), work=work)
    within(o, ref, bound, "o")


# --------------------------------------------------------- as they are used together
def _decode_step(dtype, n=3, hq=8, hkv=2, dim=128, cap=300):
    """The operators of one generated token: norms and rotation of q and k, the new row into the
    cache, attention over it."""
    g = dict(qg=1 + 0.1 * rnd(20, 1, dim).cuda(), kg=1 + 0.1 * rnd(21, 1, dim).cuda())
    s = dict(x=rnd(22, n, hq + 2 * hkv, dim, dtype=dtype).cuda(), rope=R.rope_table(cap, dim).cuda(),
             pos=torch.tensor([299, 0, 57], dtype=torch.int32, device="cuda"), cache=_cache(n, hkv, cap, dim), **g)
    old_k, old_v = rnd(23, n * cap, hkv, dim, dtype=dtype).cuda(), rnd(24, n * cap, hkv, dim, dtype=dtype).cuda()
    B.cs_kv4_store(s["cache"], old_k, old_v)
    s["slots"] = (torch.arange(n, device="cuda") * cap).int() + s["pos"]
    s["lens"] = s["pos"] + 1
    q, k = s["x"][:, :hq], s["x"][:, hq:hq + hkv]
    s["q"] = torch.empty(n, hq, dim, dtype=dtype, device="cuda")
    s["k"] = torch.empty(n, hkv, dim, dtype=dtype, device="cuda")
    s["o"] = torch.empty(n, 1, hq, dim, dtype=dtype, device="cuda")
    nd = B.qk_norm_desc(q, k, s["q"], s["k"], s["qg"], s["kg"], s["rope"], style=B.CS_ROPE_HALVES)
    ad = B.kv4_attn_desc(s["q"].view(n, 1, hq, dim), s["cache"], s["o"])
    need = B.cs_kv4_attention_workspace(ad)
    work = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        B.cs_qk_norm_rope(nd, q, k, s["q"], s["k"], s["qg"], s["kg"], s["rope"], s["pos"], stream)
        B.cs_kv4_store(s["cache"], s["k"], s["x"][:, hq + hkv:], s["slots"], stream)
        B.cs_kv4_attention(ad, s["q"].view(n, 1, hq, dim), s["cache"], s["o"], None, s["lens"], None, work, stream)
    return s, step


@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_token_through_norm_cache_and_attention(dtype):
    s, step = _decode_step(dtype)
    step()
    torch.cuda.synchronize()
    n, hq, dim = s["q"].shape
    hkv = s["k"].shape[1]
    x, at = s["x"], s["pos"].long().cpu()
    for got, src, gain in ((s["q"], x[:, :hq], s["qg"]), (s["k"], x[:, hq:hq + hkv], s["kg"])):
        ref, mag = R.norm_rope(src, gain, s["rope"], at, True, 1e-6)
        within(got, ref, R.norm_bound(mag, dim, dtype), "norm")
    t = [c.cpu() for c in s["cache"].tensors]
    for i, src in ((0, s["k"]), (2, x[:, hq + hkv:])):
        c, b = R.quantise(src)
        assert torch.equal(t[i][torch.arange(n), :, at], c) and torch.equal(t[i + 1][torch.arange(n), :, at], b)
    k, v = (R.dequantise(t[i], t[i + 1]).transpose(1, 2) for i in (0, 2))
    ref, bound = R.attention(s["q"].view(n, 1, hq, dim), k, v, 1 / math.sqrt(dim), None, s["lens"].cpu(), None, dtype == BF)
    within(s["o"], ref, bound, "o")


@pytest.mark.parametrize("dtype", [BF, FP])
def test_captured_and_replayed(dtype):
    s, step = _decode_step(dtype)
    step()
    torch.cuda.synchronize()
    want = s["o"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    x0 = s["x"].clone()
    for i in range(4):
        s["x"].copy_(x0 * (1 + i))          # eager work of the program between replays
        s["o"].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = s["o"].clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, s["o"]), i
        if i == 0:
            assert torch.equal(got, want)


def test_two_streams_with_a_workspace_each():
    pairs = [_decode_step(BF) for _ in range(2)]
    pairs[1][0]["x"].mul_(-1.5)
    want = []
    for s, step in pairs:
        step()
        torch.cuda.synchronize()
        want.append(s["o"].clone())
        s["o"].zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for (s, step), st in zip(pairs, streams):
            step(st)
    torch.cuda.synchronize()
    for (s, _), w in zip(pairs, want):
        assert torch.equal(s["o"], w)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_without_a_stream_calls_go_to_the_current_one(dtype):
    """Behind what torch enqueued on it, and into a graph that is being captured on it."""
    s, step = _decode_step(dtype)
    x0 = s["x"].clone()
    step()
    torch.cuda.synchronize()
    want = s["o"].clone()
    a = rnd(5, 2048, 2048).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s["x"].fill_(9.0)
        for _ in range(100):            # a while, behind which the input comes
            a = a @ a * 1e-3
        s["x"].copy_(x0)
        step()
        got = s["o"].clone()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for scale in (2.0, -1.0, 1.0):
        s["x"].copy_(scale * x0)
        s["o"].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = s["o"].clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, s["o"])
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_two_graphs_that_share_a_workspace(dtype):
    """One after the other on one stream: a workspace carries nothing from call to call.  Joined
    parts of keys, unpacked rows (bf16) and shapes of more than a round of workgroups."""
    lens = torch.tensor([1200, 0, 700], dtype=torch.int32, device="cuda")
    calls = []
    for seed, (lq, kv4) in enumerate([(2, False), (2, True), (300, True), (1100, False)]):
        q = rnd(seed, 3, lq, 8, 128, dtype=dtype).cuda()
        k, v = rnd(10 + seed, 3, 1200, 8, 128, dtype=dtype).cuda(), rnd(20 + seed, 3, 1200, 8, 128, dtype=dtype).cuda()
        o = torch.empty_like(q)
        if kv4:
            cache = _cache(3, 8, 1200, 128)
            B.cs_kv4_store(cache, k.flatten(0, 1), v.flatten(0, 1))
            d = B.kv4_attn_desc(q, cache, o)
            need = B.cs_kv4_attention_workspace(d)
            call = lambda w, st=None, d=d, q=q, c=cache, o=o: B.cs_kv4_attention(d, q, c, o, None, lens, None, w, st)
        else:
            d = B.attn_desc(q, k, v, o)
            need = B.cs_cross_attention_workspace(d)
            call = lambda w, st=None, d=d, q=q, k=k, v=v, o=o: B.cs_cross_attention(d, q, k, v, o, None, lens, None, w, st)
        calls.append((call, o, need))
    work = torch.empty(max(1, max(need for _, _, need in calls)), dtype=torch.uint8, device="cuda")
    want, graphs, side = [], [], torch.cuda.Stream()
    for call, o, need in calls:
        call(torch.empty(max(1, need), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        want.append(o.clone())
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(work, side)
        graphs.append(graph)
    for i in range(3):
        for _, o, _ in calls:
            o.fill_(7.0)
        work.random_(0, 256)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, o, _), w in zip(calls, want):
            assert torch.equal(o, w), i
