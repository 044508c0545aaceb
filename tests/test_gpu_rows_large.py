"""Large calls of layer norm, rows in 8 bits and their product: what fits a launch is not refused, and what only
large calls do (sums over long groups, accesses past the caches) is compared."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import rows_ref as R
from paper_2607_23159_amd import binding as B
from test_gpu_layer_norm import BF, FP, padded, run_grad, within


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
