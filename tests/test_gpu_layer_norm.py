"""Layer norm by itself, forward (to bf16, fp32 and 8 bits) and backward, against float64, at the
sizes and layouts where it can go wrong."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import rows_ref as R
from paper_2607_23159_amd import binding as B

BF, FP, I8 = torch.bfloat16, torch.float32, torch.int8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def rnd(seed, *shape, scale=1.0):
    return scale * torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def padded(rows, dim, dtype, fill, extra=0):
    """A [rows][dim] tensor whose rows lie on 16 bytes inside a larger one, and a check that the rest
    still holds `fill`."""
    unit = 16 // torch.empty(0, dtype=dtype).element_size()
    wide = (dim + unit - 1) // unit * unit + extra * unit
    whole = torch.full((rows + 8, wide), fill, dtype=dtype, device="cuda")
    t = whole[4:4 + rows, :dim]

    def check():
        rest = whole.clone()
        rest[4:4 + rows, :dim] = fill
        assert (rest == fill).all(), "written out of bounds"
    return t, check


def put(x, dtype, extra=0):
    t, _ = padded(*x.shape, dtype, 3, extra)
    t.copy_(x)
    return t


def within(got, ref, bound, what):
    got = got.double().cpu()
    bad = ~((got - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), "worst", float(((got - ref).abs() / bound).nan_to_num(9e9).max()),
                           "first", [int(x[0]) for x in bad.nonzero(as_tuple=True)])


def data(groups, rows, dim, xt, params, seed=0, mean=0.5):
    x = put(rnd(seed, groups * rows, dim) * (0.2 + torch.rand(dim, generator=torch.Generator().manual_seed(9))) +
            mean * rnd(seed + 1, dim), xt, extra=1)
    w = put(rnd(seed + 2, groups, dim, scale=0.4) + 0.2, FP, extra=2) if "w" in params else None
    b = put(rnd(seed + 3, groups, dim, scale=0.3), FP) if "b" in params else None
    return x, w, b


SHAPES = [  # groups, rows, dim: lanes, chunks and waves that are partly or just filled
    (1, 1, 1), (1, 3, 2), (2, 5, 7), (1, 1, 64), (3, 4, 100), (1, 2, 256), (1, 9, 511), (2, 3, 512), (1, 5, 513),
    (1, 6, 1536), (3, 297, 256), (1, 4, 2047), (1, 7, 2048), (2, 3, 2049), (1, 3, 5120), (1, 2, 8192), (2, 2, 8200),
    (2, 2, 8960), (2, 1, 12287), (2, 2, 12288), (1, 2, 13824), (1, 3, 16383), (1, 1, 16384),
]
TYPES = [(BF, BF), (BF, FP), (FP, BF), (FP, FP)]


@pytest.mark.parametrize("xt,yt", TYPES)
@pytest.mark.parametrize("groups,rows,dim", SHAPES)
def test_forward(groups, rows, dim, xt, yt):
    for params, unit in (("wb", False), ("wb", True), ("w", True), ("b", False), ("", False)):
        x, w, b = data(groups, rows, dim, xt, params)
        y, check = padded(groups * rows, dim, yt, -77.0, extra=2)
        mean, rstd = torch.empty(groups * rows, device="cuda"), torch.empty(groups * rows, device="cuda")
        d = B.layer_norm_desc(x, y, w, b, groups=groups, unit_offset=unit, eps=1e-5)
        B.cs_layer_norm(d, x, y, w, b, mean=mean, rstd=rstd)
        ref, off, m, m_off, r, r_rel = R.layer_norm(x, w, b, groups, unit, 1e-5)
        within(y, ref, off + R.HALF[yt] * (ref.abs() + off), (params, unit))
        within(mean, m, m_off, "mean")
        within(rstd, r, r * r_rel, "rstd")
        check()


@pytest.mark.parametrize("xt", [BF, FP])
@pytest.mark.parametrize("groups,rows,dim", SHAPES)
def test_forward_to_8_bits(groups, rows, dim, xt):
    """The codes are those of the fp32 result, exactly."""
    x, w, b = data(groups, rows, dim, xt, "wb")
    full, _ = padded(groups * rows, dim, FP, 0.0)
    B.cs_layer_norm(B.layer_norm_desc(x, full, w, b, groups=groups, unit_offset=True), x, full, w, b)
    q, check = padded(groups * rows, dim, I8, 55, extra=1)
    s = torch.empty(groups * rows, device="cuda")
    B.cs_layer_norm(B.layer_norm_desc(x, q, w, b, groups=groups, unit_offset=True), x, q, w, b, y_scale=s)
    codes, scales = R.to_codes(full)
    assert torch.equal(s.cpu(), scales) and torch.equal(q.cpu(), codes)
    check()


def test_forward_of_constant_huge_and_non_finite_rows():
    dim = 300
    x = rnd(1, 8, dim)
    x[0] = 4.5                       # no variance
    x[1] = 0.0
    x[2] = 1e30 * rnd(2, dim)        # squares overflow: rstd 0, the bias is left
    x[3, 7] = math.nan
    x[4, 299] = math.inf
    x[5] = 1e-25 * rnd(3, dim)
    x[6] = 3.0e4 + 1e-2 * rnd(4, dim)   # far from zero
    xd = put(x, FP)
    w, b = put(rnd(5, 1, dim), FP), put(rnd(6, 1, dim), FP)
    for yt in (FP, BF, I8):
        y, check = padded(8, dim, yt, 11)
        s = torch.zeros(8, device="cuda")
        rstd = torch.empty(8, device="cuda")
        d = B.layer_norm_desc(xd, y, w, b)
        B.cs_layer_norm(d, xd, y, w, b, y_scale=s, rstd=rstd)
        check()
        back = y.float() if yt != I8 else y.float() * s[:, None]
        back = back.double().cpu()
        assert torch.isnan(back[3]).all() and torch.isnan(back[4]).all() and rstd[2] == 0
        if yt == I8:
            assert (y[3] == 0).all() and (y[4] == 0).all() and torch.isnan(s[3:5]).all()
            continue
        bias = b.double().cpu()[0]
        for row in (0, 1, 2):
            within(back[row], bias, R.HALF[yt] * bias.abs(), row)
        ok = torch.tensor([0, 1, 5, 6, 7])
        ref, off = R.layer_norm(x[ok], w, b, 1, False, 1e-6)[:2]
        within(back[ok], ref, off + R.HALF[yt] * (ref.abs() + off), "finite rows")


@pytest.mark.parametrize("xt", [BF, FP])
def test_forward_in_place_and_independent_of_the_batch(xt):
    for dim in (40, 1536, 5120):
        x, w, b = data(3, 17, dim, xt, "wb")
        y, _ = padded(51, dim, xt, 0.0)
        d = B.layer_norm_desc(x, y, w, b, groups=3)
        B.cs_layer_norm(d, x, y, w, b)
        x2 = x.clone()
        x2 = put(x, xt, extra=1)
        B.cs_layer_norm(B.layer_norm_desc(x2, x2, w, b, groups=3), x2, x2, w, b)
        assert torch.equal(x2, y)
        one, _ = padded(1, dim, xt, 0.0)
        for g, r in ((0, 0), (1, 3), (2, 16)):
            xs, ws, bs = x[17 * g + r:17 * g + r + 1], w[g:g + 1], b[g:g + 1]
            B.cs_layer_norm(B.layer_norm_desc(xs, one, ws, bs), xs, one, ws, bs)
            assert torch.equal(one[0], y[17 * g + r])


def test_rows_past_32_bits():
    """Rows whose elements lie past 2^31 elements and 2^32 bytes of the first."""
    rows, dim, stride = 5, 64, 1 << 29
    whole = torch.empty(4 * stride + 64, dtype=BF, device="cuda")
    x = torch.as_strided(whole, (rows, dim), (stride, 1))
    x.copy_(rnd(0, rows, dim))
    d = B.layer_norm_desc(x, x)
    ref, off = R.layer_norm(x, None, None, 1, False, 1e-6)[:2]
    B.cs_layer_norm(d, x, x)
    within(x, ref, off + R.HALF[BF] * (ref.abs() + off), "rows")
    xs = x.clone()
    q = torch.as_strided(whole.view(I8)[:], (rows, dim), (2 * stride, 1))
    s = torch.empty(rows, device="cuda")
    codes, scales = R.to_codes(xs)
    B.cs_i8_quantise(B.i8_rows_desc(xs, q, s), xs, q, s)
    assert torch.equal(q.cpu(), codes) and torch.equal(s.cpu(), scales)


@pytest.mark.parametrize("dim", [1536, 2051])
def test_large_calls_are_those_of_their_parts(dim):
    """Calls of more than 384 MB read and write past the caches: bitwise the same, forward, in 8 bits and
    back, and backward."""
    groups, rows = 6, 8000
    total = groups * rows
    x, _ = padded(total, dim, FP, 0.0)
    x.copy_(torch.randn(total, dim, generator=torch.Generator("cuda").manual_seed(1), device="cuda"))
    w, b = put(rnd(2, groups, dim), FP), put(rnd(3, groups, dim), FP)
    y, check_y = padded(total, dim, FP, -77.0, extra=1)
    mean, rstd = torch.empty(total, device="cuda"), torch.empty(total, device="cuda")
    B.cs_layer_norm(B.layer_norm_desc(x, y, w, b, groups=groups), x, y, w, b, mean=mean, rstd=rstd)
    q, check_q = padded(total, dim, I8, 55)
    s = torch.empty(total, device="cuda")
    B.cs_i8_quantise(B.i8_rows_desc(x, q, s), x, q, s)
    back, check_back = padded(total, dim, FP, -77.0)
    B.cs_i8_dequantise(B.i8_rows_desc(back, q, s), q, s, back)
    t = run_grad(x, y, w, mean, rstd, groups, True)
    for g in (0, 2, 5):
        r = slice(g * rows, (g + 1) * rows)
        one, wg, bg = padded(rows, dim, FP, 0.0)[0], w[g:g + 1], b[g:g + 1]
        m, d = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        B.cs_layer_norm(B.layer_norm_desc(x[r], one, wg, bg), x[r], one, wg, bg, mean=m, rstd=d)
        assert torch.equal(one, y[r]) and torch.equal(m, mean[r]) and torch.equal(d, rstd[r])
        q1, s1 = padded(rows, dim, I8, 0)[0], torch.empty(rows, device="cuda")
        B.cs_i8_quantise(B.i8_rows_desc(x[r], q1, s1), x[r], q1, s1)
        assert torch.equal(q1, q[r]) and torch.equal(s1, s[r])
        B.cs_i8_dequantise(B.i8_rows_desc(one, q1, s1), q1, s1, one)
        assert torch.equal(one, back[r])
        p = run_grad(x[r], y[r], wg, m, d, 1, True)
        assert torch.equal(p["x"], t["x"][r]) and torch.equal(p["w"][0], t["w"][g]) and torch.equal(p["b"][0], t["b"][g])
    for check in (check_y, check_q, check_back):
        check()


# ---------------------------------------------------------------------- backward
def grad_case(groups, rows, dim, xt, dyt, unit, with_w=True, seed=0):
    x, w, _ = data(groups, rows, dim, xt, "w" if with_w else "", seed)
    dy = put(rnd(seed + 7, groups * rows, dim), dyt)
    m = x.double().mean(-1)
    rstd = (1.0 / torch.sqrt(((x.double() - m[:, None]) ** 2).mean(-1) + 1e-6)).float()
    return x, dy, w, m.float(), rstd


def run_grad(x, dy, w, mean, rstd, groups, unit, want="xwb", stream=None):
    rows, dim = x.shape
    out = {}
    if "x" in want:
        out["x"] = padded(rows, dim, x.dtype, -77.0, extra=1)
    for k in "wb":
        if k in want:
            out[k] = padded(groups, dim, FP, -77.0, extra=3)
    t = {k: v[0] for k, v in out.items()}
    d = B.layer_norm_grad_desc(x, dy, w, t.get("x"), t.get("w"), t.get("b"), groups=groups, unit_offset=unit)
    need = B.cs_layer_norm_backward_workspace(d)
    work = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")   # NaN
    B.cs_layer_norm_backward(d, x, dy, w, mean, rstd, t.get("x"), t.get("w"), t.get("b"), work=work, stream=stream)
    for _, check in out.values():
        check()
    return t


GRADS = SHAPES + [(1, 16, 100), (1, 32, 101), (2, 32, 5121), (1, 33, 100), (4, 33, 2050), (2, 32, 1536), (2, 600, 40), (1, 8300, 24), (5, 33, 1536), (2, 40, 5120)]


@pytest.mark.parametrize("xt,dyt", TYPES)
@pytest.mark.parametrize("groups,rows,dim", GRADS)
def test_backward(groups, rows, dim, xt, dyt):
    for unit, with_w in ((False, True), (True, True), (False, False)):
        x, dy, w, mean, rstd = grad_case(groups, rows, dim, xt, dyt, unit, with_w)
        if dim == 1:
            rstd.fill_(0.75)       # a row of one channel has no variance: any statistics do
        t = run_grad(x, dy, w, mean, rstd, groups, unit)
        (dx, off), dw, db = R.layer_norm_grad(x, dy, w, mean, rstd, groups, unit)
        within(t["x"], dx, off + R.HALF[xt] * (dx.abs() + off), "dx")
        within(t["w"], *dw, "dw")
        within(t["b"], *db, "db")
        for want in ("x", "w", "b", "wb"):
            s = run_grad(x, dy, w, mean, rstd, groups, unit, want)
            assert all(torch.equal(s[k], t[k]) for k in want), want


def test_backward_against_differences():
    """dx, dw and db of sum(c y) by central differences of the float64 formula."""
    groups, rows, dim = 2, 3, 50
    x, dy, w, mean, rstd = grad_case(groups, rows, dim, FP, FP, True, seed=40)
    b = put(rnd(60, groups, dim), FP)
    t = run_grad(x, dy, w, mean, rstd, groups, True)
    c = dy.double().cpu()

    def loss(xx, ww, bb):
        return (R.layer_norm(xx, ww, bb, groups, True, 1e-6)[0] * c).sum()
    base = [v.double().cpu() for v in (x, w, b)]
    for k, name in enumerate("xwb"):
        for at in ((0, 0), (1, 49), (0, 17)):
            h = 1e-5
            side = []
            for s in (h, -h):
                v = [p.clone() for p in base]
                v[k][at] += s
                side.append(loss(*v))
            slope = float((side[0] - side[1]) / (2 * h))
            # the formula's third derivatives times h^2, and fp32's rounding of sums of 50 and 6 terms
            assert abs(float(t[name][at]) - slope) <= 2e-5 * max(1.0, abs(slope)), (name, at)


def test_backward_of_no_rows_and_of_groups_alone():
    x, dy, w, mean, rstd = grad_case(1, 0, 24, FP, FP, False)
    w = put(rnd(1, 1, 24), FP)
    t = run_grad(x, dy, w, mean, rstd, 1, False)
    assert (t["w"] == 0).all() and (t["b"] == 0).all()
    for dim, rows in ((256, 297), (1536, 70), (2100, 20)):
        x, dy, w, mean, rstd = grad_case(3, rows, dim, FP, BF, True)
        t = run_grad(x, dy, w, mean, rstd, 3, True)
        for g in range(3):
            r = slice(g * rows, (g + 1) * rows)
            s = run_grad(x[r], dy[r], w[g:g + 1], mean[r].clone(), rstd[r].clone(), 1, True)
            assert torch.equal(s["x"], t["x"][r]) and torch.equal(s["w"][0], t["w"][g]) and torch.equal(s["b"][0], t["b"][g])


@pytest.mark.parametrize("dim", [1, 100, 101, 1536, 5000, 5001])
def test_backward_of_rows_far_from_zero(dim):
    """Channels that a row does not have must not count: their n would be -mean rstd, past fp32 here."""
    x, dy, w, mean, rstd = grad_case(1, 5, dim, FP, FP, False)
    x.fill_(1e37)
    mean.fill_(1e37)
    rstd.fill_(1000.0)
    t = run_grad(x, dy, w, mean, rstd, 1, False)
    (dx, off), dw, db = R.layer_norm_grad(x, dy, w, mean, rstd, 1, False)
    within(t["x"], dx, off + R.HALF[FP] * (dx.abs() + off), "dx")
    within(t["w"], *dw, "dw")
    within(t["b"], *db, "db")


@pytest.mark.parametrize("dim", [96, 5120])
def test_backward_in_place(dim):
    x, dy, w, mean, rstd = grad_case(2, 21, dim, BF, BF, False)
    t = run_grad(x, dy, w, mean, rstd, 2, False)
    for k in range(2):
        a = [put(x, BF, extra=1), put(dy, BF)]
        dx = a[k]
        d = B.layer_norm_grad_desc(a[0], a[1], w, dx, groups=2)
        B.cs_layer_norm_backward(d, a[0], a[1], w, mean, rstd, dx)
        assert torch.equal(dx, t["x"])


def test_norms_in_a_graph_and_on_another_stream():
    groups, rows, dim = 2, 37, 640
    x, dy, w, mean, rstd = grad_case(groups, rows, dim, FP, BF, True)
    b = put(rnd(9, groups, dim), FP)
    y = torch.empty(groups * rows, dim, dtype=BF, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    df = B.layer_norm_desc(x, y, w, b, groups=groups, unit_offset=True)
    dg = B.layer_norm_grad_desc(x, dy, w, dx, dw, db, groups=groups, unit_offset=True)
    work = torch.empty(B.cs_layer_norm_backward_workspace(dg), dtype=torch.uint8, device="cuda")

    def call(stream=None):
        B.cs_layer_norm(df, x, y, w, b, mean=mean, rstd=rstd, stream=stream)
        B.cs_layer_norm_backward(dg, x, dy, w, mean, rstd, dx, dw, db, work=work, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (11, 12, 13):
        x.copy_(rnd(seed, groups * rows, dim))
        dy.copy_(rnd(seed + 50, groups * rows, dim))
        call()
        want = [t.clone() for t in (y, dx, dw, db)]
        for t in (y, dx, dw, db, mean, rstd):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, t) for a, t in zip(want, (y, dx, dw, db)))


@pytest.mark.parametrize("groups,rows,dim", [(1, 40, 130), (3, 33, 1536), (2, 19, 5120)])
def test_forward_then_backward_is_the_gradient(groups, rows, dim):
    """The kept statistics lead to the gradient that float64's own differentiation gives."""
    x, w, b = data(groups, rows, dim, FP, "wb", seed=70)
    dy = put(rnd(77, groups * rows, dim), FP)
    y, mean, rstd = padded(groups * rows, dim, FP, 0.0)[0], *(torch.empty(groups * rows, device="cuda") for _ in range(2))
    B.cs_layer_norm(B.layer_norm_desc(x, y, w, b, groups=groups, unit_offset=True), x, y, w, b, mean=mean, rstd=rstd)
    t = run_grad(x, dy, w, mean, rstd, groups, True)
    leaves = [v.double().cpu().requires_grad_() for v in (x, w, b)]
    out = torch.nn.functional.layer_norm(leaves[0], (dim,), eps=1e-6).reshape(groups, rows, dim)
    out = out * (1.0 + leaves[1])[:, None] + leaves[2][:, None]
    out.backward(dy.double().cpu().reshape(out.shape))
    # what the kernel is off by for its statistics, and what they are off by themselves: m rstd and rel of
    # layer_norm's bound, through n and the factor rstd
    (_, off), (_, w_off), (_, b_off) = R.layer_norm_grad(x, dy, w, mean, rstd, groups, True)
    m, rel = R.layer_norm(x, w, b, groups, True, 1e-6)[3::2]
    r = rstd.double().cpu()
    stat = (m * r + 2 * rel)[:, None]                       # of n, relative to 1 + |n|
    n = (x.double().cpu() - mean.double().cpu()[:, None]) * r[:, None]
    g = dy.double().cpu() * (1.0 + w.double().cpu().repeat_interleave(rows, 0))
    more = r[:, None] * stat * 4 * ((1 + n.abs()) * (g * n).abs().mean(-1, keepdim=True) + g.abs().mean(-1, keepdim=True) + g.abs() +
                                    n.abs() * (g.abs() * (1 + n.abs())).mean(-1, keepdim=True))
    grad = [v.grad for v in leaves]
    within(t["x"], grad[0], off + more + R.HALF[FP] * grad[0].abs(), "dx")
    w_more = (dy.double().cpu().abs() * stat * (1 + n.abs())).reshape(groups, rows, dim).sum(1)
    within(t["w"], grad[1], w_off + 1.01 * w_more, "dw")
    within(t["b"], grad[2], b_off, "db")


def test_two_graphs_that_share_a_workspace():
    """One after the other, in either order: a workspace carries nothing over."""
    runs = []
    work = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    for groups, rows, dim in ((2, 70, 640), (1, 300, 1000)):
        x, dy, w, mean, rstd = grad_case(groups, rows, dim, BF, BF, False, seed=dim)
        dw, db = torch.empty(groups, dim, device="cuda"), torch.empty(groups, dim, device="cuda")
        d = B.layer_norm_grad_desc(x, dy, w, None, dw, db, groups=groups)
        assert B.cs_layer_norm_backward_workspace(d) <= work.numel()

        def call(d=d, x=x, dy=dy, w=w, mean=mean, rstd=rstd, dw=dw, db=db):
            B.cs_layer_norm_backward(d, x, dy, w, mean, rstd, None, dw, db, work=work)
        call()
        want = dw.clone(), db.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        runs.append((graph, (dw, db), want, call))     # what a graph reads has to live as long
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        for i in order:
            for t in runs[i][1]:
                t.fill_(9.0)
            runs[i][0].replay()
        torch.cuda.synchronize()
        for i in order:
            assert all(torch.equal(a, b) for a, b in zip(runs[i][1], runs[i][2]))
