"""Large calls of layer norm, rows in 8 bits and their product: what fits a launch is not refused, and what only
large calls do (sums over long groups, accesses past the caches) is compared."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import rows_ref as R
from paper_2607_23159_amd import binding as B
from test_gpu_layer_norm import BF, FP, I8, padded, run_grad, within


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()
    yield
    torch.cuda.empty_cache()


def device_randn(seed, *shape, dtype=FP):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=dtype)


# ---------------------------------------------------------------------- many groups
def many_groups(groups, rows, dim, seed=0):
    """Gradient inputs in bf16, and the float64 result of one group."""
    x, dy = (padded(groups * rows, dim, BF, 0.0)[0] for _ in range(2))
    x.copy_(device_randn(seed, groups * rows, dim, dtype=BF))
    dy.copy_(device_randn(seed + 1, groups * rows, dim, dtype=BF))
    mean, rstd = 0.1 * device_randn(seed + 2, groups * rows), 0.5 + torch.rand(groups * rows, device="cuda")
    w = padded(1, dim, FP, 0.0)[0]
    w.copy_(device_randn(seed + 3, 1, dim))
    weight = w.expand(groups, dim)         # one weight for all groups

    def ref(g):
        r = slice(g * rows, (g + 1) * rows)
        return R.layer_norm_grad(x[r], dy[r], w, mean[r], rstd[r], 1, True)
    return x, dy, weight, mean, rstd, ref


def test_gradient_of_many_groups_of_one_row():
    """A modulation for every token: the sums need no second launch, whose grid would not hold them."""
    groups, dim = 70000, 4100
    assert groups * ((dim + 63) // 64) * 1024 >= 1 << 32
    x, dy, w, mean, rstd, ref = many_groups(groups, 1, dim)
    t = run_grad(x, dy, w, mean, rstd, groups, True)
    for g in (0, 52429, groups - 1):
        (dx, off), (dw, w_off), (db, b_off) = ref(g)
        within(t["x"][g:g + 1], dx, off + R.HALF[BF] * (dx.abs() + off), "dx")
        within(t["w"][g:g + 1], dw, w_off, "dw")
        within(t["b"][g:g + 1], db, b_off, "db")


def test_gradient_of_the_rows_alone():
    """Only dx is wanted: no sums, and no launch that joins them."""
    groups, rows, dim = 1 << 22, 33, 2
    assert groups * ((dim + 63) // 64) * 1024 >= 1 << 32
    x, dy, w, mean, rstd, ref = many_groups(groups, rows, dim, seed=10)
    t = run_grad(x, dy, w, mean, rstd, groups, True, want="x")
    for g in (0, 3000001, groups - 1):
        dx, off = ref(g)[0]
        within(t["x"][g * rows:(g + 1) * rows], dx, off + R.HALF[BF] * (dx.abs() + off), "dx")


# ------------------------------------------------------------------------ long groups
def test_gradients_of_a_long_group():
    """The bound of the sums over rows, 316 half steps of fp32, holds at any length.  Every row adds the same value, 1 +
    1023 steps, which a sum between 2048 and 4096 takes as 1: 4096 rows in one fp32 sum would lose 1023 steps in half of
    them, 1024 half steps of the sum."""
    rows, dim, value = 1 << 23, 8, 1.0 + 1023 * 2.0 ** -23
    x, dy = (torch.full((rows, dim), v, device="cuda") for v in (1.0, value))
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")     # so that n is 1
    t = run_grad(x, dy, None, mean, rstd, 1, False, want="wb")
    bound = 1.01 * (300 + 16) * R.U * rows * value
    for k in "wb":
        within(t[k], torch.full((1, dim), rows * value, dtype=torch.float64), bound, k)


@pytest.mark.parametrize("rows,dim", [(131073, 24), (200001, 2056)])
def test_backward_of_groups_past_131072_rows(rows, dim):
    """As the shorter groups, against float64 (on the GPU, in slices)."""
    x, dy, _, mean, rstd, _ = many_groups(1, rows, dim, seed=20)
    t = run_grad(x, dy, None, mean, rstd, 1, False, want="wb")
    sums = torch.zeros(4, dim, dtype=torch.float64, device="cuda")
    for r in range(0, rows, 20000):
        p = slice(r, r + 20000)
        d = dy[p].double()
        dn = d * (x[p].double() - mean[p].double()[:, None]) * rstd[p].double()[:, None]
        sums += torch.stack([dn.sum(0), dn.abs().sum(0), d.sum(0), d.abs().sum(0)])
    dw, dw_abs, db, db_abs = sums.cpu()[:, None]
    within(t["w"], dw, 1.01 * (316 + 4) * R.U * dw_abs, "dw")
    within(t["b"], db, 1.01 * 316 * R.U * db_abs, "db")


# ------------------------------------------------------------------------- products
@pytest.mark.parametrize("m,n,k", [(59 * 32760, 8960, 64), (1 << 30, 7, 16)])
def test_products_of_more_outputs_than_small_tiles_cover(m, n, k):
    """Sizes whose 32 x 32 tiles (in the second case those that the costs ask for too) pass a launch's 2^32 work items,
    in larger tiles; slices are bitwise what they are alone."""
    assert -(-m // 32) * -(-n // 32) * 256 >= 1 << 32
    w = B.I8Weight(n, k)
    wq = padded(n, k, I8, 0)[0]
    wq.copy_(torch.randint(-128, 128, (n, k), device="cuda", dtype=torch.int32))
    B.cs_i8_weight_pack(w, wq, torch.rand(n, device="cuda") / 64)
    a = torch.empty(m, k, dtype=I8, device="cuda").random_(-128, 128, generator=torch.Generator("cuda").manual_seed(2))
    s = torch.rand(m, device="cuda") / 64
    o = torch.full((m, (n + 7) // 8 * 8), -77.0, dtype=BF, device="cuda")
    out = o[:, :n]
    d = B.matmul_i8_desc(a, s, w, out)
    assert B.cs_matmul_i8_workspace(d) == 0
    B.cs_matmul_i8(d, a, s, w, out)
    for first, rows in ((0, 300), (m // 2 // 4 * 4, 513), (m - 256 - m % 4, 256 + m % 4)):
        r = slice(first, first + rows)
        part = padded(rows, n, BF, 0.0)[0]
        B.cs_matmul_i8(B.matmul_i8_desc(a[r], s[r], w, part), a[r], s[r], w, part)
        assert torch.equal(part, out[r]), first
    assert (o[:, n:] == -77.0).all() and not (out[::1021] == -77.0).any()


# ------------------------------------------------------------- accesses past the caches
PAST = 384e6      # bytes of a call from which on it reads and writes past the caches


def streamed(rows, dim, *tensors):
    assert sum(rows * dim * t.element_size() for t in tensors) > PAST, "the call would stay in the caches"


def same(a, b):
    return torch.equal(a.nan_to_num(7.5e8) if a.is_floating_point() else a, b.nan_to_num(7.5e8) if b.is_floating_point() else b)


@pytest.mark.parametrize("xt", [BF, FP])
@pytest.mark.parametrize("rows,dim", [(96000, 1536), (72000, 2051), (8000, 17000)])
def test_rows_in_8_bits_past_the_caches(rows, dim, xt):
    """To codes and back, in one call and in calls that stay in the caches: bitwise the same."""
    rows *= 1 if xt == FP or dim == 17000 else 2
    x, _ = padded(rows, dim, xt, 0.0)
    for r in range(0, rows, 16000):
        n = min(16000, rows - r)
        x[r:r + n] = device_randn(r, n, dim, dtype=xt)
    x[3], x[rows - 2, dim - 1], x[rows // 2, 0] = 0.0, float("nan"), float("inf")
    q, check_q = padded(rows, dim, I8, 55, extra=1)
    s = torch.empty(rows, device="cuda")
    streamed(rows, dim, x, q)
    B.cs_i8_quantise(B.i8_rows_desc(x, q, s), x, q, s)
    back, check_back = padded(rows, dim, xt, -77.0, extra=1)
    B.cs_i8_dequantise(B.i8_rows_desc(back, q, s), q, s, back)
    step = 4000
    q1, s1, back1 = padded(step, dim, I8, 0)[0], torch.empty(step, device="cuda"), padded(step, dim, xt, 0.0)[0]
    for first in range(0, rows, step):
        p = slice(first, first + step)
        B.cs_i8_quantise(B.i8_rows_desc(x[p], q1, s1), x[p], q1, s1)
        assert same(q1, q[p]) and same(s1, s[p]), first
        B.cs_i8_dequantise(B.i8_rows_desc(back1, q1, s1), q1, s1, back1)
        assert same(back1, back[p]), first
    check_q()
    check_back()


@pytest.mark.parametrize("xt,yt", [(BF, BF), (BF, FP), (FP, BF), (BF, I8), (FP, I8)])
@pytest.mark.parametrize("dim", [1536, 2051, 5120])
def test_norms_past_the_caches(dim, xt, yt):
    """Forward, and backward with gradients of the forward's type."""
    groups, rows = 4, 64 * (-(-100_000_000 // (dim * (torch.empty(0, dtype=xt).element_size() + torch.empty(0, dtype=yt).element_size())))
                            // 64 + 1)
    total = groups * rows
    x, _ = padded(total, dim, xt, 0.0)
    x.copy_(device_randn(1, total, dim, dtype=xt))
    w, b = padded(groups, dim, FP, 0.0)[0], padded(groups, dim, FP, 0.0)[0]
    w.copy_(device_randn(2, groups, dim))
    b.copy_(device_randn(3, groups, dim))
    y, check = padded(total, dim, yt, 55 if yt == I8 else -77.0, extra=1)
    mean, rstd, s = (torch.empty(total, device="cuda") for _ in range(3))
    streamed(total, dim, x, y)
    B.cs_layer_norm(B.layer_norm_desc(x, y, w, b, groups=groups), x, y, w, b, y_scale=s, mean=mean, rstd=rstd)
    t = None
    if yt != I8:
        streamed(total, dim, x, y, x)
        t = run_grad(x, y, w, mean, rstd, groups, True)
    for g in range(groups):
        r, wg, bg = slice(g * rows, (g + 1) * rows), w[g:g + 1], b[g:g + 1]
        one = padded(rows, dim, yt, 0)[0]
        m, d, s1 = (torch.empty(rows, device="cuda") for _ in range(3))
        B.cs_layer_norm(B.layer_norm_desc(x[r], one, wg, bg), x[r], one, wg, bg, y_scale=s1, mean=m, rstd=d)
        assert same(one, y[r]) and same(m, mean[r]) and same(d, rstd[r]) and (yt != I8 or same(s1, s[r]))
        if t is not None:
            p = run_grad(x[r], y[r], wg, m, d, 1, True)
            assert same(p["x"], t["x"][r]) and same(p["w"][0], t["w"][g]) and same(p["b"][0], t["b"][g])
    check()
