"""What layer norm, rows in 8 bits and their product refuse, before any device work (no GPU
needed), and what their binding refuses and hands on."""
import ctypes as C
import math

import pytest

from paper_2607_23159_amd import binding as B

P = 1 << 20        # an aligned address that no refused call touches
BIG = 2 ** 31 - 1


def refused(status, name, word):
    assert status == getattr(B, "CS_E_" + name), (status, B.cs_last_error())
    assert word in B.cs_last_error(), B.cs_last_error()


# ------------------------------------------------------------------ layer norm
def norm_desc(**kw):
    d = dict(x_dtype=B.CS_FP32, y_dtype=B.CS_BF16, groups=2, rows=3, dim=40, unit_offset=0, eps=1e-6, x_row=40, y_row=40,
             w_group=40, b_group=40)
    d.update(kw)
    return B.cs_layer_norm_desc(**d)


def norm(d, x=P, w=P, b=P, y=P, s=None, mean=None, rstd=None):
    return B.lib().cs_layer_norm(None if d is None else C.byref(d), x, w, b, y, s, mean, rstd, None)


def grad_desc(**kw):
    d = dict(x_dtype=B.CS_FP32, y_dtype=B.CS_BF16, groups=2, rows=3, dim=40, unit_offset=0, x_row=40, dy_row=40, dx_row=40,
             w_group=40, dw_group=40, db_group=40)
    d.update(kw)
    return B.cs_layer_norm_grad_desc(**d)


def grad(d, x=P, dy=P, w=P, mean=P, rstd=P, dx=P, dw=P, db=P, work=P, nbytes=1 << 40):
    return B.lib().cs_layer_norm_backward(None if d is None else C.byref(d), x, dy, w, mean, rstd, dx, dw, db, work, nbytes,
                                          None)


COMMON = [
    (dict(x_dtype=B.CS_I8), "INVAL", "x_dtype"), (dict(x_dtype=-1), "INVAL", "x_dtype"), (dict(groups=-1), "INVAL", "groups"),
    (dict(rows=-1), "INVAL", "rows"), (dict(groups=1 << 16, rows=1 << 14), "UNSUPPORTED", "2^30"),
    (dict(groups=BIG, rows=BIG), "UNSUPPORTED", "2^30"), (dict(dim=0), "INVAL", "dim"), (dict(dim=-8), "INVAL", "dim"),
    (dict(dim=16385), "UNSUPPORTED", "dim"), (dict(unit_offset=2), "INVAL", "unit_offset"),
    (dict(w_group=2), "INVAL", "w_group"), (dict(w_group=-4), "INVAL", "w_group"), (dict(x_row=41), "INVAL", "x_row"),
    (dict(x_row=-40), "INVAL", "x_row"), (dict(x_row=1 << 60), "UNSUPPORTED", "x_row"),
    (dict(x_dtype=B.CS_BF16, x_row=44), "INVAL", "x_row"),
]


@pytest.mark.parametrize("kw,status,word", COMMON + [
    (dict(y_dtype=3), "INVAL", "y_dtype"), (dict(eps=-1e-9), "INVAL", "eps"), (dict(eps=math.nan), "INVAL", "eps"),
    (dict(eps=math.inf), "INVAL", "eps"), (dict(b_group=6), "INVAL", "b_group"), (dict(y_row=44), "INVAL", "y_row"),
    (dict(y_row=0), "INVAL", "y_row"), (dict(y_dtype=B.CS_I8, y_row=40), "INVAL", "y_row")])
def test_norm_descriptors(kw, status, word):
    refused(norm(norm_desc(**kw)), status, word)


def test_norm_pointers_and_nothing_to_do():
    refused(norm(None), "INVAL", "NULL")
    for name in ("x", "y"):
        refused(norm(norm_desc(), **{name: None}), "INVAL", name)
    for name in ("x", "y", "w", "b", "mean", "rstd"):
        refused(norm(norm_desc(), **{name: P + 4}), "INVAL", "aligned")
    i8 = norm_desc(y_dtype=B.CS_I8, y_row=48)
    refused(norm(i8), "INVAL", "y_scale")
    refused(norm(i8, s=P + 4), "INVAL", "y_scale")
    for kw in (dict(groups=0), dict(rows=0)):
        assert norm(norm_desc(**kw), x=None, y=None, w=None, b=None) == B.CS_OK


@pytest.mark.parametrize("kw,status,word", COMMON + [
    (dict(y_dtype=B.CS_I8), "INVAL", "y_dtype"), (dict(dy_row=4), "INVAL", "dy_row"), (dict(dx_row=2), "INVAL", "dx_row"),
    (dict(dx_row=0), "INVAL", "output stride"), (dict(dw_group=0), "INVAL", "dw_group"),
    (dict(db_group=2), "INVAL", "db_group")])
def test_norm_grad_descriptors(kw, status, word):
    refused(grad(grad_desc(**kw)), status, word)


def test_norm_grad_pointers_workspace_and_nothing_to_do():
    refused(grad(None), "INVAL", "NULL")
    for name in ("x", "dy", "mean", "rstd"):
        refused(grad(grad_desc(), **{name: None}), "INVAL", name)
    for name in ("x", "dy", "w", "mean", "rstd", "dx", "dw", "db"):
        refused(grad(grad_desc(), **{name: P + 4}), "INVAL", "aligned")
    fn, n = B.lib().cs_layer_norm_backward_workspace, C.c_size_t(77)
    assert fn(C.byref(grad_desc()), None) == B.CS_E_INVAL
    assert fn(C.byref(grad_desc(dim=0)), C.byref(n)) == B.CS_E_INVAL and n.value == 77
    for kw in (dict(rows=33), dict(rows=300), dict(groups=1, rows=100000, dim=16384)):
        assert fn(C.byref(grad_desc(**kw)), C.byref(n)) == B.CS_OK and 0 < n.value < 1 << 31
    for rows in (0, 1, 32):
        assert fn(C.byref(grad_desc(rows=rows)), C.byref(n)) == B.CS_OK and n.value == 0
    assert fn(C.byref(grad_desc(rows=70)), C.byref(n)) == B.CS_OK
    for kw in (dict(work=None), dict(work=P + 8), dict(nbytes=n.value - 1)):
        for only in (dict(), dict(dx=None, dw=None), dict(db=None)):
            refused(grad(grad_desc(rows=70), **kw, **only), "INVAL", "workspace")
    assert grad(grad_desc(), dx=None, dw=None, db=None, work=None, nbytes=0) == B.CS_OK
    assert grad(grad_desc(groups=0), x=None, dy=None, work=None) == B.CS_OK
    # the part of a group does not depend on how many groups there are
    one = C.c_size_t(0)
    for rows in (1, 15, 16, 17, 300, 8192, 8193, 32760, 262080):
        assert fn(C.byref(grad_desc(groups=1, rows=rows)), C.byref(one)) == B.CS_OK
        assert fn(C.byref(grad_desc(groups=5, rows=rows)), C.byref(n)) == B.CS_OK
        assert n.value == 5 * one.value


# ---------------------------------------------------------------------- 8 bits
def rows(**kw):
    d = dict(dtype=B.CS_BF16, rows=3, dim=40, x_row=40, q_row=48)
    d.update(kw)
    return B.cs_i8_rows(**d)


@pytest.mark.parametrize("store", [True, False])
def test_rows(store):
    def go(r, x=P, q=P, s=P):
        r = None if r is None else C.byref(r)
        return B.lib().cs_i8_quantise(r, x, q, s, None) if store else B.lib().cs_i8_dequantise(r, q, s, x, None)
    refused(go(None), "INVAL", "NULL")
    for kw, status, word in ((dict(dtype=B.CS_I8), "INVAL", "dtype"), (dict(rows=-1), "INVAL", "rows"),
                             (dict(dim=0), "INVAL", "dim"), (dict(dim=65537), "UNSUPPORTED", "dim"),
                             (dict(x_row=44), "INVAL", "x_row"), (dict(q_row=40), "INVAL", "q_row"),
                             (dict(q_row=-48), "INVAL", "q_row"), (dict(q_row=1 << 60), "UNSUPPORTED", "q_row"),
                             (dict(q_row=0) if store else dict(x_row=0), "INVAL", "output stride")):
        refused(go(rows(**kw)), status, word)
    for name in ("x", "q", "s"):
        refused(go(rows(), **{name: None}), "INVAL", "NULL")
        refused(go(rows(), **{name: P + 4}), "INVAL", "aligned")
    assert go(rows(rows=0), x=None, q=None, s=None) == B.CS_OK


def weight(**kw):
    d = dict(codes=P, scales=P, n=24, k=40)
    d.update(kw)
    return B.cs_i8_weight(**d)


BAD_WEIGHTS = [(dict(n=0), "INVAL", "n and k"), (dict(k=0), "INVAL", "n and k"), (dict(n=(1 << 24) + 1), "UNSUPPORTED", "2^24"),
               (dict(k=65537), "UNSUPPORTED", "65536"), (dict(codes=None), "INVAL", "codes"),
               (dict(codes=P + 8), "INVAL", "aligned"), (dict(scales=None), "INVAL", "scales"),
               (dict(scales=P + 4), "INVAL", "aligned")]


def test_weights():
    fn, n = B.lib().cs_i8_weight_bytes, C.c_size_t(77)
    for a in ((0, 1), (1, 0), (-1, 5)):
        assert fn(*a, C.byref(n)) == B.CS_E_INVAL and n.value == 77
    assert fn(1, 1, None) == B.CS_E_INVAL
    for a, want in (((1, 1), 256 * 128), ((256, 128), 256 * 128), ((257, 129), 512 * 256), ((1 << 24, 65536), 1 << 40)):
        assert fn(*a, C.byref(n)) == B.CS_OK and n.value == want

    def go(o, dtype=B.CS_FP32, w=P, row=40, s=None):
        return B.lib().cs_i8_weight_pack(None if o is None else C.byref(o), dtype, w, row, s, None)
    refused(go(None), "INVAL", "NULL")
    for kw, status, word in BAD_WEIGHTS:
        refused(go(weight(**kw)), status, word)
    refused(go(weight(), dtype=3), "INVAL", "dtype")
    refused(go(weight(), row=42), "INVAL", "w_row")
    refused(go(weight(), w=None), "INVAL", "NULL")
    refused(go(weight(), s=P), "INVAL", "w_scales")
    refused(go(weight(), dtype=B.CS_I8, row=48), "INVAL", "w_scales")
    refused(go(weight(), dtype=B.CS_I8, row=40, s=P), "INVAL", "w_row")


def mm_desc(**kw):
    d = dict(out_dtype=B.CS_BF16, rows=5, n=24, k=40, act=0, a_row=48, o_row=24)
    d.update(kw)
    return B.cs_matmul_i8_desc(**d)


def mm(d, a=P, s=P, w="default", b=None, o=P, work=None, nbytes=0):
    w = weight() if w == "default" else w
    return B.lib().cs_matmul_i8(None if d is None else C.byref(d), a, s, None if w is None else C.byref(w), b, o, work, nbytes,
                                None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(out_dtype=B.CS_I8), "INVAL", "out_dtype"), (dict(rows=-1), "INVAL", "rows"),
    (dict(rows=(1 << 30) + 1), "UNSUPPORTED", "2^30"), (dict(n=0), "INVAL", "n and k"), (dict(k=-1), "INVAL", "n and k"),
    (dict(k=70000), "UNSUPPORTED", "65536"), (dict(act=2), "INVAL", "act"), (dict(a_row=40), "INVAL", "a_row"),
    (dict(a_row=(1 << 22) + 16), "UNSUPPORTED", "a_row"), (dict(o_row=20), "INVAL", "o_row"),
    (dict(o_row=0), "INVAL", "output stride"),
    (dict(n=25), "INVAL", "weight's"), (dict(k=39), "INVAL", "weight's")])
def test_product_descriptors(kw, status, word):
    refused(mm(mm_desc(**kw)), status, word)


def test_product_pointers_workspace_and_nothing_to_do():
    refused(mm(None), "INVAL", "NULL")
    refused(mm(mm_desc(), w=None), "INVAL", "NULL")
    for kw, status, word in BAD_WEIGHTS:
        refused(mm(mm_desc(), w=weight(**kw)), status, word)
    for name in ("a", "s", "o"):
        refused(mm(mm_desc(), **{name: None}), "INVAL", "NULL")
    for name in ("a", "s", "o", "b"):
        refused(mm(mm_desc(), **{name: P + 4}), "INVAL", "aligned")
    assert mm(mm_desc(rows=0), a=None, s=None, o=None) == B.CS_OK
    fn, n = B.lib().cs_matmul_i8_workspace, C.c_size_t(77)
    assert fn(C.byref(mm_desc()), None) == B.CS_E_INVAL
    assert fn(C.byref(mm_desc(act=9)), C.byref(n)) == B.CS_E_INVAL and n.value == 77
    for r, cols, k in ((1, 64, 65536), (5, 24, 40), (100, 1536, 8960), (40000, 24, 40)):
        d, w = mm_desc(rows=r, n=cols, k=k, a_row=65536, o_row=1536), weight(n=cols, k=k)
        assert fn(C.byref(d), C.byref(n)) == B.CS_OK and n.value < 1 << 34
        if n.value:
            for kw in (dict(), dict(work=P, nbytes=n.value - 1), dict(work=P + 8, nbytes=n.value)):
                refused(mm(d, w=w, **kw), "INVAL", "workspace")


# --------------------------------------------------------------------- binding
torch = pytest.importorskip("torch")
from test_ops_binding import CURRENT, DEV, _desc, recorder  # noqa: E402,F401


def test_binding_refuses_host_tensors_and_other_types():
    x, q, s = torch.zeros(4, 16), torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    for call in (lambda: B.layer_norm_desc(x, x), lambda: B.layer_norm_grad_desc(x, x, dx=x), lambda: B.i8_rows_desc(x, q, s)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    for call in (lambda: B.layer_norm_desc(x.half(), x), lambda: B.i8_rows_desc(x.double(), q, s)):
        with pytest.raises(ValueError, match="bfloat16 or float32"):
            call()
    for bad in (s, s.double(), torch.zeros(3)):
        with pytest.raises(ValueError):
            B._vector(bad, 4, "scales", DEV)
    assert B._vector(s, 4, "scales", s.device) == s.data_ptr()
    with pytest.raises(ValueError):
        B._vector(torch.zeros(8)[::2], 4, "scales", s.device)
    with pytest.raises(ValueError, match="3 groups"):
        B._norm_rows(x, 3)
    with pytest.raises(ValueError, match="without it"):
        B._given(x, None, "bias")
    with pytest.raises(ValueError, match="with it"):
        B._given(None, B._sig(x), "bias")


def test_operators_run_on_the_current_stream_or_the_given_one(recorder):  # noqa: F811
    class Stream:
        cuda_stream = 77

    class FakeWeight:
        device, ref = DEV, C.byref(B.cs_i8_weight())
    n = _desc(B.cs_layer_norm_desc(groups=1, rows=1), "x", "y", "weight", "bias")
    g = _desc(B.cs_layer_norm_grad_desc(groups=1, rows=1), "x", "dy", "weight", "dx", "dweight", "dbias")
    r = _desc(B.cs_i8_rows(), "x", "codes", "scales")
    m = _desc(B.cs_matmul_i8_desc(n=1), "codes", "scales", "out")
    for stream, want in ((None, CURRENT), (Stream(), 77), (0, 0)):
        kw = {} if stream is None else dict(stream=stream)
        recorder.calls.clear()
        B.cs_layer_norm(n, P, P, P, P, **kw)
        B.cs_layer_norm_backward(g, P, P, P, P, P, P, P, P, **kw)
        B.cs_i8_quantise(r, P, P, P, **kw)
        B.cs_i8_dequantise(r, P, P, P, **kw)
        B.cs_matmul_i8(m, P, P, FakeWeight(), P, **kw)
        assert [c[0] for c in recorder.calls] == ["cs_layer_norm", "cs_layer_norm_backward", "cs_i8_quantise",
                                                  "cs_i8_dequantise", "cs_matmul_i8"]
        assert [args[-1] for _, args in recorder.calls] == [want] * 5


def test_calls_too_large_for_a_grid():
    """A launch has fewer than 2^32 work items."""
    wide = dict(groups=1, rows=1 << 24, dim=4096, x_row=4096)
    refused(norm(norm_desc(y_row=4096, **wide)), "UNSUPPORTED", "too many")
    refused(norm(norm_desc(groups=1, rows=1 << 27, x_row=40, y_row=40)), "UNSUPPORTED", "too many")
    refused(grad(grad_desc(groups=1 << 24, rows=1), nbytes=1 << 60), "UNSUPPORTED", "too many")
    refused(grad(grad_desc(groups=1 << 18, rows=0, dim=1024, w_group=1024, dw_group=1024, db_group=1024)), "UNSUPPORTED",
            "too many")
    for kw in (dict(rows=1 << 24, dim=4096, x_row=4096, q_row=4096), dict(rows=1 << 27, dim=16, x_row=16, q_row=16),
               dict(rows=1 << 22, dim=20000, x_row=20000, q_row=20000)):
        r = C.byref(rows(**kw))
        refused(B.lib().cs_i8_quantise(r, P, P, P, None), "UNSUPPORTED", "too many")
        if kw["dim"] != 20000:
            refused(B.lib().cs_i8_dequantise(r, P, P, P, None), "UNSUPPORTED", "too many")
    refused(mm(mm_desc(rows=1 << 30, n=1 << 14, o_row=1 << 14), w=weight(n=1 << 14)), "UNSUPPORTED", "too many")


def test_projections_in_8_bits_refuse_fp32_and_unknown_formats():
    from paper_2607_23159_amd import synth
    out = C.c_void_p()
    m = synth.MODELS["tiny"]
    n = synth.weight_count(m)

    def go(dtype, proj, w=P, count=n):
        return B.lib().cs_model_init_proj(C.byref(B.model_desc(m, dtype)), 0, proj, w, count, None, C.byref(out))
    refused(go(B.CS_FP32, B.CS_PROJ_8BIT), "UNSUPPORTED", "CS_BF16")
    refused(go(B.CS_BF16, 2), "INVAL", "proj")
    refused(go(B.CS_BF16, -1), "INVAL", "proj")
    refused(go(B.CS_I8, B.CS_PROJ_8BIT), "INVAL", "dtype")
    refused(go(B.CS_BF16, B.CS_PROJ_8BIT, w=None), "INVAL", "weights")
    refused(go(B.CS_BF16, B.CS_PROJ_8BIT, count=n - 1), "INVAL", "expected")
