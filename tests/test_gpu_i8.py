"""Rows in 8 bits and back, 8-bit weights, and their product, against exact integers and float64."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import rows_ref as R
from paper_2607_23159_amd import binding as B
from test_gpu_layer_norm import BF, FP, I8, padded, put, rnd, within


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


# ------------------------------------------------------------------------- rows
@pytest.mark.parametrize("xt", [BF, FP])
@pytest.mark.parametrize("rows,dim", [(1, 1), (2, 3), (5, 16), (1, 100), (3, 512), (4, 513), (9, 1536), (3, 2048), (2, 2052),
                                      (2, 5120), (3, 8192), (2, 8960), (1, 16384), (2, 16385), (1, 40000), (2, 65536)])
def test_rows_to_8_bits_and_back(rows, dim, xt):
    x = put(rnd(rows + dim, rows, dim) * (0.1 + rnd(3, dim).abs()), xt, extra=1)
    q, check_q = padded(rows, dim, I8, 55, extra=1)
    s = torch.empty(rows, device="cuda")
    B.cs_i8_quantise(B.i8_rows_desc(x, q, s), x, q, s)
    codes, scales = R.to_codes(x)
    assert torch.equal(s.cpu(), scales) and torch.equal(q.cpu(), codes)
    check_q()
    back, check = padded(rows, dim, xt, -77.0, extra=2)
    B.cs_i8_dequantise(B.i8_rows_desc(back, q, s), q, s, back)
    assert torch.equal(back.cpu(), (codes.float() * scales[:, None]).to(xt))
    check()


def test_rounding_next_to_halfway_values():
    """Quotients on and next to every halfway value, for scales of many mantissas."""
    for seed in range(8):
        top = (1.0 + torch.rand(64, generator=torch.Generator().manual_seed(seed))).float() * 2.0 ** (7 * seed - 20)
        s = (top.double() / 127).float()
        half = (torch.arange(-127, 127).double() + 0.5)[None] * s.double()[:, None]
        x = half.float()
        x = torch.cat([x, torch.nextafter(x, torch.tensor(math.inf)), torch.nextafter(x, torch.tensor(-math.inf)),
                       s[:, None] * torch.arange(-127, 128).float()], 1).clamp(-top[:, None], top[:, None])
        x = torch.cat([x, top[:, None]], 1)
        xd = put(x, FP)
        q, _ = padded(*x.shape, I8, 0)
        sd = torch.empty(64, device="cuda")
        B.cs_i8_quantise(B.i8_rows_desc(xd, q, sd), xd, q, sd)
        codes, scales = R.to_codes(x)
        assert torch.equal(sd.cpu(), scales) and torch.equal(q.cpu(), codes)
    # scales of one mantissa bit: exact halves
    x = torch.cat([torch.arange(-254, 255).float() / 2, torch.tensor([127.0])])[None].repeat(3, 1)
    x[1] *= 2.0 ** -60
    x[2] *= 2.0 ** 90
    xd = put(x, FP)
    q, _ = padded(*x.shape, I8, 0)
    sd = torch.empty(3, device="cuda")
    B.cs_i8_quantise(B.i8_rows_desc(xd, q, sd), xd, q, sd)
    assert torch.equal(q.cpu(), R.to_codes(x)[0])


def test_rows_of_zeros_tiny_huge_and_non_finite_values():
    dim = 700
    x = rnd(1, 12, dim)
    x[0] = 0.0
    x[1] = -0.0
    x[2] *= 1e-38
    x[3] *= 1e-43                    # the scale is a few units of the smallest number
    x[4] = 1e-45                     # and here it underflows
    x[5] *= 8e37
    x[6] = torch.finfo(FP).max
    x[7, 699], x[8, 0], x[9, 333] = math.nan, math.inf, -math.inf
    x[10] = 0.0
    x[10, 5] = -3.0
    for xt in (FP, BF):
        xd = put(x, xt)
        q, check = padded(12, dim, I8, 55)
        s = torch.empty(12, device="cuda")
        B.cs_i8_quantise(B.i8_rows_desc(xd, q, s), xd, q, s)
        check()
        codes, scales = R.to_codes(xd)
        assert torch.equal(q.cpu(), codes)
        assert torch.equal(s.cpu().nan_to_num(-1.0), scales.nan_to_num(-1.0))
        assert torch.isnan(s[7:10]).all() if xt == FP else torch.isnan(s[7]).all()
        back, _ = padded(12, dim, xt, 0.0)
        B.cs_i8_dequantise(B.i8_rows_desc(back, q, s), q, s, back)
        assert torch.isnan(back[7:10]).all() and (back[:2] == 0).all() and back[10, 5] == -3.0


# ------------------------------------------------------------------------ product
def weight_of(n, k, seed=0, dtype=I8):
    """(packed weight, codes, scales)"""
    w = rnd(seed, n, k) * (0.3 + rnd(seed + 1, n, 1).abs()) / math.sqrt(k)
    o = B.I8Weight(n, k)
    if dtype == I8:
        q, s = R.to_codes(w)
        q = torch.where(torch.rand(n, k, generator=torch.Generator().manual_seed(seed)) < 1e-3, -128, q.int()).to(I8)
        B.cs_i8_weight_pack(o, put(q, I8, extra=1), s.cuda())
        return o, q, s
    wd = put(w, dtype, extra=1)
    B.cs_i8_weight_pack(o, wd)
    return o, *R.to_codes(wd)


def rows_of(m, k, seed=0):
    q, s = R.to_codes(rnd(seed, m, k) * (0.1 + rnd(seed + 1, k).abs()))
    q = torch.where(torch.rand(m, k, generator=torch.Generator().manual_seed(seed)) < 1e-3, -128, q.int()).to(I8)
    t, _ = padded(m, k, I8, 113, extra=seed % 3)     # what lies past k is not zero
    t.copy_(q)
    return t, s.cuda()


def product(a, s, w, out_type, bias=None, act=False, extra=1):
    o, check = padded(a.shape[0], w.c.n, out_type, -77.0, extra=extra)
    d = B.matmul_i8_desc(a, s, w, o, act=B.CS_ACT_GELU if act else B.CS_ACT_NONE)
    need = B.cs_matmul_i8_workspace(d)
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    B.cs_matmul_i8(d, a, s, w, o, bias=bias, work=work)
    check()
    return o


MM = [  # rows, n, k
    (1, 1, 1), (1, 16, 128), (1, 5, 17), (2, 3, 100), (1, 1536, 256), (3, 130, 127), (7, 33, 129), (16, 64, 1536),
    (17, 64, 130), (31, 257, 300), (32, 512, 512), (33, 31, 640), (64, 64, 128), (65, 100, 1000), (100, 1000, 65),
    (128, 128, 4096), (129, 255, 1030), (200, 700, 333), (257, 513, 256), (300, 96, 8960), (511, 2049, 70),
    (891, 512, 256), (1, 300, 13824), (5, 260, 65536), (1030, 1540, 200), (2100, 300, 390), (64, 5000, 140),
    (4200, 1100, 80), (16, 4096, 70), (16, 4097, 70), (17, 4096, 70), (9, 4000, 1100),
    # in parts of K
    (17, 512, 8960), (33, 70, 9000), (64, 300, 13824), (100, 515, 6300), (300, 513, 8961), (16, 4100, 16000), (40, 33, 65536),
]


@pytest.mark.parametrize("out_type", [BF, FP])
@pytest.mark.parametrize("m,n,k", MM)
def test_product(m, n, k, out_type):
    w, wq, ws = weight_of(n, k, seed=n)
    a, s = rows_of(m, k, seed=m + k)
    bias = rnd(5, n, scale=0.5).cuda()
    for b, act in ((None, False), (bias, False), (bias, True)):
        o = product(a, s, w, out_type, b, act)
        ref, off = R.matmul(a, s, wq, ws, b, act)
        within(o, ref, off + R.HALF[out_type] * (ref.abs() + off), (b is not None, act))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n,k", [(1, 1), (3, 40), (257, 130), (64, 1536), (300, 2000)])
def test_weights_from_values(n, k, dtype):
    w, wq, ws = weight_of(n, k, seed=3, dtype=dtype)
    assert torch.equal(w.tensors[1].cpu(), ws)
    # unit rows read the codes back
    eye = torch.zeros(k, k, dtype=I8)
    eye.fill_diagonal_(1)
    a = put(eye, I8)
    one = torch.ones(k, device="cuda")
    got = product(a, one, w, FP)
    assert torch.equal(got.cpu(), (wq.float() * ws[:, None]).t().contiguous())


def test_product_does_not_depend_on_the_batch_or_the_kernel():
    for n, k in ((70, 200), (1536, 512), (640, 5120), (130, 9000)):
        w, _, _ = weight_of(n, k)
        bias = rnd(1, n).cuda()
        a, s = rows_of(1300, k, seed=4)
        for t, act in ((BF, True), (FP, False)):
            whole = product(a, s, w, t, bias, act)
            for first, rows in ((0, 1), (1299, 1), (5, 3), (100, 16), (17, 17), (40, 40), (600, 65), (300, 129), (10, 700)):
                part = product(a[first:first + rows], s[first:first + rows].clone(), w, t, bias, act)
                assert torch.equal(part, whole[first:first + rows]), (n, k, first, rows)


def test_scales_that_are_zero_nan_or_extreme():
    w, wq, ws = weight_of(90, 64)
    a, s = rows_of(9, 64)
    bias = rnd(1, 90).cuda()
    s[0], s[1], s[2], s[3] = 0.0, math.nan, 1e30, 1e-38
    o = product(a, s, w, FP, bias)
    assert torch.equal(o[0], bias) and torch.isnan(o[1]).all()
    ref, off = R.matmul(a[2:], s[2:], wq, ws, bias, False)
    within(o[2:], ref, off, "extreme")
    g = product(a, s, w, FP, bias, True)
    assert torch.isnan(g[1]).all() and not torch.isnan(g[[0, 2, 3, 4, 5]]).any()


def test_a_row_stride_larger_than_the_rows_and_rows_at_the_end_of_memory():
    k, n = 200, 96
    w, wq, ws = weight_of(n, k)
    whole = torch.randint(-128, 128, (40, 4096), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(I8).cuda()
    s = torch.rand(40, device="cuda")
    for col in (0, 16, 4096 - 208):
        a = whole[:, col:col + k]
        o = product(a, s, w, FP)
        ref, off = R.matmul(a, s, wq, ws, None, False)
        within(o, ref, off, col)


def test_a_norm_in_8_bits_then_its_product_in_a_graph():
    """The run of the operators together: norm with modulation, codes, product with GELU."""
    groups, rows, dim, n = 2, 45, 384, 700
    x = put(rnd(0, groups * rows, dim), FP)
    w, b = put(0.2 * rnd(1, groups, dim), FP), put(0.2 * rnd(2, groups, dim), FP)
    q = torch.empty(groups * rows, dim, dtype=I8, device="cuda")
    s = torch.empty(groups * rows, device="cuda")
    weight, wq, ws = weight_of(n, dim)
    bias = rnd(3, n).cuda()
    o, check = padded(groups * rows, n, BF, -77.0)
    dn = B.layer_norm_desc(x, q, w, b, groups=groups, unit_offset=True)
    dm = B.matmul_i8_desc(q, s, weight, o, act=B.CS_ACT_GELU)
    need = B.cs_matmul_i8_workspace(dm)
    work = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")

    def call():
        B.cs_layer_norm(dn, x, q, w, b, y_scale=s)
        B.cs_matmul_i8(dm, q, s, weight, o, bias=bias, work=work)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    full = torch.empty(groups * rows, dim, device="cuda")
    for seed in (5, 6, 7):
        x.copy_(rnd(seed, groups * rows, dim))
        call()
        want = o.clone()
        B.cs_layer_norm(B.layer_norm_desc(x, full, w, b, groups=groups, unit_offset=True), x, full, w, b)
        codes, scales = R.to_codes(full)
        ref, off = R.matmul(codes, scales, wq, ws, bias, True)
        within(want, ref, off + R.HALF[BF] * (ref.abs() + off), "chain")
        o.fill_(1.0)
        q.fill_(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
    check()


def test_products_on_two_streams_at_once():
    w, _, _ = weight_of(1536, 1536)
    a, s = rows_of(700, 1536)
    want = product(a, s, w, BF)
    sides = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty(700, 1536, dtype=BF, device="cuda") for _ in sides]
    d = B.matmul_i8_desc(a, s, w, outs[0])
    works = [torch.empty(max(1, B.cs_matmul_i8_workspace(d)), dtype=torch.uint8, device="cuda") for _ in sides]
    torch.cuda.synchronize()
    for _ in range(4):
        for st, o, k in zip(sides, outs, works):
            B.cs_matmul_i8(d, a, s, w, o, work=k, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


# Shapes that the choices give each of the tiles (test_i8_tile_choice.py), whole and in parts of K, odd in
# every direction.
TILES = {"W4_256x256": (7000, 4330, 930), "W4_224x256": (6265, 1818, 924), "W4_192x256": (1305, 8018, 553),
         "W4_160x256": (4104, 2273, 417), "W4_128x128": (1740, 3589, 132), "W4_64x64": (3013, 65, 100),
         "RING_128x128": (7184, 417, 514), "RING_64x128": (4499, 200, 1821), "RING_64x64": (38, 8454, 1236),
         "RING_32x64": (17, 3325, 101), "RING_32x32": (17, 17, 103)}
PARTS = {"RING_64x128": (38, 5330, 12175), "RING_64x64": (33, 1581, 8752), "RING_32x64": (33, 2156, 6061),
         "RING_32x32": (17, 17, 6395)}


@pytest.mark.parametrize("m,n,k", [*TILES.values(), *PARTS.values()])
def test_product_in_every_tile(m, n, k):
    """The integer sums are exact; what is made of them rounds twice on the way and once at the end."""
    g = torch.Generator("cuda").manual_seed(m)
    a, wq = padded(m, k, I8, 0)[0], padded(n, k, I8, 0)[0]
    for t in (a, wq):
        t.copy_(torch.randint(-128, 128, t.shape, generator=g, device="cuda", dtype=torch.int32))
    s, ws = torch.rand(m, generator=g, device="cuda") / 64, torch.rand(n, generator=g, device="cuda") / 64
    bias = torch.randn(n, generator=g, device="cuda")
    w = B.I8Weight(n, k)
    B.cs_i8_weight_pack(w, wq, ws)
    p = (a.double() @ wq.double().t().contiguous()) * s.double()[:, None] * ws.double()
    ref = p + bias.double()
    off = 2 * R.U * p.abs() + R.U * ref.abs()
    del p
    for t in (FP, BF):
        o = product(a, s, w, t, bias)
        bad = (o.double() - ref).abs() > 1.01 * off + R.HALF[t] * (ref.abs() + off) + 1e-37
        assert not bad.any(), (t, int(bad.sum()), [int(x[0]) for x in bad.nonzero(as_tuple=True)])


@pytest.mark.parametrize("m,n,k,stride", [(600, 130, 200, 1 << 22), (3013, 65, 100, 1 << 21), (33, 70, 9000, 1 << 22)])
def test_rows_past_32_bits(m, n, k, stride):
    """Rows of codes and outputs that lie past 2^31 bytes and elements of the first (600, 3,013 rows)."""
    w, wq, ws = weight_of(n, k)
    whole = torch.empty((m - 1) * stride + 4096 * 4, dtype=I8, device="cuda")
    a = torch.as_strided(whole, (m, k), (stride, 1))
    q, s = rows_of(m, k)
    a.copy_(q)
    out = torch.empty((m - 1) * stride + 4096, dtype=BF, device="cuda")
    o = torch.as_strided(out, (m, n), (stride, 1))
    d = B.matmul_i8_desc(a, s, w, o)
    work = torch.empty(max(1, B.cs_matmul_i8_workspace(d)), dtype=torch.uint8, device="cuda")
    B.cs_matmul_i8(d, a, s, w, o, work=work)
    assert torch.equal(o, product(q, s, w, BF))


def test_graphs_that_share_a_workspace_of_parts():
    w1, _, _ = weight_of(300, 9000)
    w2, _, _ = weight_of(500, 13824)
    runs, work = [], None
    for w, m in ((w1, 40), (w2, 64)):
        a, s = rows_of(m, w.c.k, seed=m)
        o = torch.empty(m, (w.c.n + 7) // 8 * 8, dtype=BF, device="cuda")[:, :w.c.n]
        d = B.matmul_i8_desc(a, s, w, o)
        assert B.cs_matmul_i8_workspace(d) > 0
        work = torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda") if work is None else work
        B.cs_matmul_i8(d, a, s, w, o, work=work)
        want = o.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.cs_matmul_i8(d, a, s, w, o, work=work)
        runs.append((graph, o, want, a, s))     # what a graph reads has to live as long
    for order in ((0, 1), (1, 0), (0, 0)):
        for i in order:
            runs[i][1].fill_(9.0)
            runs[i][0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(runs[i][1], runs[i][2]) for i in order)
