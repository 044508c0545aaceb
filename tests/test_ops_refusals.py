"""What the stand-alone operators refuse, before any device work (no GPU needed)."""
import ctypes as C
import math

import pytest

from paper_2607_23159_amd import binding as B

P = 1 << 20        # an aligned address that no refused call touches


def norm_desc(**kw):
    d = dict(dtype=B.CS_BF16, tokens=4, heads_q=2, heads_k=1, head_dim=64, rot_dim=64, rope_rows=8, rope_style=0,
             eps=1e-6, q_row=128, q_head=64, k_row=64, k_head=64, qo_row=128, qo_head=64, ko_row=64, ko_head=64,
             q_gain_head=0, k_gain_head=0)
    d.update(kw)
    return B.cs_qk_norm_desc(**d)


def norm(d, q=P, k=P, qo=P, ko=P, qg=P, kg=P, rope=P, pos=None):
    return B.lib().cs_qk_norm_rope(None if d is None else C.byref(d), q, k, qo, ko, qg, kg, rope, pos, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=2), "INVAL", "dtype"), (dict(tokens=-1), "INVAL", "tokens"), (dict(heads_k=-1), "INVAL", "heads"),
    (dict(head_dim=8), "INVAL", "head_dim"), (dict(head_dim=72), "UNSUPPORTED", "head_dim"),
    (dict(head_dim=272), "UNSUPPORTED", "head_dim"), (dict(rot_dim=80), "INVAL", "rot_dim"),
    (dict(rot_dim=24), "UNSUPPORTED", "rot_dim"), (dict(rot_dim=-16), "INVAL", "rot_dim"),
    (dict(rope_rows=0), "INVAL", "rope_rows"), (dict(rope_style=2), "INVAL", "rope_style"),
    (dict(eps=-1.0), "INVAL", "eps"), (dict(eps=math.nan), "INVAL", "eps"), (dict(eps=math.inf), "INVAL", "eps"),
    (dict(q_row=-128), "INVAL", "q_row"), (dict(q_head=60), "INVAL", "q_head"), (dict(ko_row=2), "INVAL", "ko_row"),
    (dict(qo_row=1 << 60), "UNSUPPORTED", "qo_row"), (dict(q_gain_head=2), "INVAL", "q_gain_head"),
    (dict(tokens=2 ** 31 - 1, heads_q=2 ** 20, q_row=8, q_head=8, qo_row=8, qo_head=8), "UNSUPPORTED", "too many"),
])
def test_norm_descriptors(kw, status, word):
    assert norm(norm_desc(**kw)) == getattr(B, "CS_E_" + status)
    assert word in B.cs_last_error()


def test_norm_pointers_and_nothing_to_do():
    d = norm_desc()
    assert norm(None) == B.CS_E_INVAL
    for name in ("q", "k", "qo", "ko", "qg", "kg", "rope"):
        assert norm(d, **{name: None}) == B.CS_E_INVAL and "NULL" in B.cs_last_error()
        assert norm(d, **{name: P + 4}) == B.CS_E_INVAL and "aligned" in B.cs_last_error()
    assert norm(norm_desc(tokens=0), q=None, k=None) == B.CS_OK
    assert norm(norm_desc(heads_q=0, heads_k=0), q=None, k=None, rope=None) == B.CS_OK


def attn_desc(**kw):
    d = dict(dtype=B.CS_BF16, n_q=2, n_kv=2, lq=3, lk=40, heads_q=4, heads_kv=2, head_dim=64, scale=0.125,
             q_b=768, q_r=256, q_h=64, k_b=5120, k_r=128, k_h=64, v_b=5120, v_r=128, v_h=64, o_b=768, o_r=256, o_h=64,
             mask_b=40)
    d.update(kw)
    return B.cs_attn_desc(**d)


def attn(d, q=P, k=P, v=P, of=None, ln=None, mask=None, o=P, work=None, nbytes=0):
    return B.lib().cs_cross_attention(None if d is None else C.byref(d), q, k, v, of, ln, mask, o, work, nbytes, None)


def cache(**kw):
    c = dict(k_codes=P, k_scales=P, v_codes=P, v_scales=P, n_kv=2, heads=2, cap=40, head_dim=64)
    c.update(kw)
    return B.cs_kv4_cache(**c)


def kv4(d, c, q=P, of=None, ln=None, mask=None, o=P, work=None, nbytes=0):
    return B.lib().cs_kv4_attention(None if d is None else C.byref(d), q, None if c is None else C.byref(c), of, ln,
                                    mask, o, work, nbytes, None)


BAD_ATTN = [
    (dict(dtype=-1), "INVAL", "dtype"), (dict(n_q=-1), "INVAL", "n_q"), (dict(lq=-1), "INVAL", "lq"),
    (dict(lk=-2), "INVAL", "lk"), (dict(n_kv=0), "INVAL", "n_kv"), (dict(heads_q=0), "INVAL", "heads"),
    (dict(heads_q=3), "INVAL", "multiple"), (dict(head_dim=96), "UNSUPPORTED", "head_dim"),
    (dict(scale=0.0), "INVAL", "scale"), (dict(scale=math.nan), "INVAL", "scale"),
    (dict(scale=math.inf), "INVAL", "scale"), (dict(scale=-1.0), "INVAL", "scale"),
    (dict(mask_b=-1), "INVAL", "mask_b"), (dict(lq=1 << 30, q_r=8, o_r=8), "UNSUPPORTED", "2^30"),
    (dict(q_r=-8), "INVAL", "q_r"), (dict(q_h=4), "INVAL", "q_h"), (dict(o_b=1 << 60), "UNSUPPORTED", "o_b"),
]


@pytest.mark.parametrize("kw,status,word", BAD_ATTN + [
    (dict(k_r=132), "INVAL", "k_r"), (dict(v_h=-64), "INVAL", "v_h"), (dict(n_q=3), "INVAL", "kv_of")])
def test_cross_attention_descriptors(kw, status, word):
    assert attn(attn_desc(**kw)) == getattr(B, "CS_E_" + status)
    assert word in B.cs_last_error()


@pytest.mark.parametrize("kw,status,word", BAD_ATTN + [
    (dict(lk=39), "INVAL", "cache"), (dict(n_kv=3), "INVAL", "cache"), (dict(heads_kv=4), "INVAL", "cache"),
    (dict(head_dim=32), "INVAL", "cache")])
def test_kv4_attention_descriptors(kw, status, word):
    assert kv4(attn_desc(**kw), cache()) == getattr(B, "CS_E_" + status)
    assert word in B.cs_last_error()


def test_attention_pointers_workspaces_and_nothing_to_do():
    n = C.c_size_t(77)
    assert attn(None) == B.CS_E_INVAL and kv4(None, cache()) == B.CS_E_INVAL
    assert kv4(attn_desc(), None) == B.CS_E_INVAL
    for name in ("q", "k", "v", "o"):
        assert attn(attn_desc(), **{name: None}) == B.CS_E_INVAL and "NULL" in B.cs_last_error()
        assert attn(attn_desc(), **{name: P + 8}) == B.CS_E_INVAL and "aligned" in B.cs_last_error()
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert kv4(attn_desc(), cache(**{name: None})) == B.CS_E_INVAL
        assert kv4(attn_desc(), cache(**{name: P + 1})) == B.CS_E_INVAL
    for kw in (dict(n_q=0), dict(lq=0)):
        assert attn(attn_desc(**kw), q=None, o=None) == B.CS_OK
        assert kv4(attn_desc(**kw), cache(), q=None, o=None) == B.CS_OK
    for fn in (B.lib().cs_cross_attention_workspace, B.lib().cs_kv4_attention_workspace):
        assert fn(C.byref(attn_desc()), None) == B.CS_E_INVAL
        assert fn(C.byref(attn_desc(scale=0.0)), C.byref(n)) == B.CS_E_INVAL and n.value == 77
        assert fn(C.byref(attn_desc()), C.byref(n)) == B.CS_OK and n.value < 1 << 40
        n.value = 77


def test_a_workspace_that_is_missing_or_small_is_refused():
    d = attn_desc(lq=1, lk=1 << 20, k_b=1 << 28, v_b=1 << 28)
    n = C.c_size_t(0)
    assert B.lib().cs_cross_attention_workspace(C.byref(d), C.byref(n)) == B.CS_OK
    if n.value:
        assert attn(d) == B.CS_E_INVAL and "workspace" in B.cs_last_error()
        assert attn(d, work=P, nbytes=n.value - 1) == B.CS_E_INVAL and "workspace" in B.cs_last_error()
        assert attn(d, work=P + 8, nbytes=n.value) == B.CS_E_INVAL and "workspace" in B.cs_last_error()


def rows(**kw):
    r = dict(dtype=B.CS_BF16, n_rows=10, k_row=128, k_head=64, v_row=128, v_head=64)
    r.update(kw)
    return B.cs_kv4_rows(**r)


@pytest.mark.parametrize("call", ["cs_kv4_store", "cs_kv4_load"])
def test_rows_of_the_cache(call):
    fn = getattr(B.lib(), call)

    def go(c, r, k=P, v=P, slots=None):
        return fn(None if c is None else C.byref(c), None if r is None else C.byref(r), k, v, slots, None)

    bad = [(cache(n_kv=0), rows()), (cache(heads=-1), rows()), (cache(cap=0), rows()), (cache(k_codes=None), rows()),
           (cache(v_scales=P + 2), rows()), (cache(), rows(dtype=9)), (cache(), rows(n_rows=-1)),
           (cache(), rows(n_rows=81)), (cache(), rows(k_row=4)), (cache(), rows(v_head=-8)), (None, rows()),
           (cache(), None)]
    for c, r in bad:
        assert go(c, r) == B.CS_E_INVAL
    assert go(cache(head_dim=256), rows()) == B.CS_E_UNSUPPORTED
    assert go(cache(n_kv=1 << 16, cap=1 << 15), rows()) == B.CS_E_UNSUPPORTED
    assert go(cache(), rows(k_row=1 << 60)) == B.CS_E_UNSUPPORTED
    assert go(cache(), rows(), k=None) == B.CS_E_INVAL and go(cache(), rows(), v=P + 4) == B.CS_E_INVAL
    assert go(cache(), rows(n_rows=0), k=None, v=None) == B.CS_OK
    huge = rows(n_rows=2 ** 31 - 1, k_row=8, k_head=8, v_row=8, v_head=8)
    assert go(cache(heads=1 << 20), huge, slots=P) == B.CS_E_UNSUPPORTED


def test_binding_refuses_host_tensors_and_other_shapes():
    import torch
    x = torch.zeros(2, 4, 64)
    with pytest.raises(ValueError, match="device tensor"):
        B.qk_norm_desc(x, None, x, None, x[0], None)
    with pytest.raises(ValueError, match="both None"):
        B.qk_norm_desc(None, None, None, None, None, None)
    with pytest.raises(ValueError, match="device tensor"):
        B.attn_desc(x[None], x[None], x[None], x[None])
    with pytest.raises(ValueError, match="device tensor"):
        B.Kv4Cache(*(torch.zeros(1, 1, 4, w, dtype=torch.uint8) for w in (32, 2, 32, 2)))
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        B.attn_desc(*(x[None].half(),) * 4)
    with pytest.raises(ValueError, match="the descriptor is for"):
        B._same(x, B._sig(x[:1]), "q")
    assert B._same(x, B._sig(x), "q") == x.data_ptr() and B._same(None, None, "q") is None and B._same(16, None, "q") == 16


def test_contexts_and_norm_choice_refuse_null_and_unknown():
    from paper_2607_23159_amd import synth
    lib = B.lib()
    out = C.c_void_p()
    assert lib.cs_context_init(None, P, None, 1, 0, C.byref(out)) == B.CS_E_INVAL
    assert lib.cs_context_init(None, P, None, 1, 0, None) == B.CS_E_INVAL
    assert lib.cs_velocity_context(None, None, P, None, 1, 0.5, P + 64) == B.CS_E_INVAL
    lib.cs_context_free(None)
    m = synth.MODELS["tiny"]
    d = B.model_desc(m)
    assert lib.cs_model_init_norm(C.byref(d), 2, P, synth.weight_count(m), None, C.byref(out)) == B.CS_E_INVAL
    assert "qk_norm" in B.cs_last_error()
    assert lib.cs_model_init_norm(C.byref(d), 1, None, synth.weight_count(m), None, C.byref(out)) == B.CS_E_INVAL


def test_calls_too_large_for_a_grid():
    for kw in (dict(dtype=B.CS_FP32, n_q=1 << 20, lq=1 << 12), dict(n_q=1 << 25, lq=1),
               dict(n_q=1 << 28, lq=1 << 10)):
        assert attn(attn_desc(heads_q=2, heads_kv=2, n_kv=1, q_b=8, o_b=8, q_r=8, o_r=8, q_h=8, o_h=8, **kw),
                    of=P) == B.CS_E_UNSUPPORTED
        assert "too many" in B.cs_last_error()


def test_outputs_whose_entries_coincide():
    for kw in (dict(qo_row=0), dict(qo_head=0), dict(ko_row=0)):
        assert norm(norm_desc(**kw)) == B.CS_E_INVAL and "output stride" in B.cs_last_error()
    for kw in (dict(o_b=0), dict(o_r=0), dict(o_h=0)):
        assert attn(attn_desc(**kw)) == B.CS_E_INVAL and "output stride" in B.cs_last_error()
    lib, n = B.lib(), C.c_size_t()
    for kw in (dict(k_row=0), dict(v_row=0), dict(k_head=0), dict(v_head=0)):
        r = rows(**kw)
        assert lib.cs_kv4_load(C.byref(cache()), C.byref(r), P, P, None, None) == B.CS_E_INVAL
        assert "output stride" in B.cs_last_error()
    # of one entry, and of inputs, they may be zero
    for d in (attn_desc(n_q=1, lq=1, q_b=0, q_r=0, o_b=0, o_r=0), attn_desc(q_b=0, k_b=0, v_b=0, k_h=0)):
        assert lib.cs_cross_attention_workspace(C.byref(d), C.byref(n)) == B.CS_OK


def test_sizes_whose_products_pass_64_bits():
    big = 2 ** 31 - 1
    lib, n = B.lib(), C.c_size_t(77)
    for kw, word in ((dict(n_q=big, heads_q=big - 7, heads_kv=big - 7, lq=big // 2), "too many"),
                     (dict(n_q=big, heads_q=2 ** 20, heads_kv=2 ** 20, lq=1), "too many")):
        d = attn_desc(q_b=8, q_r=8, q_h=8, o_b=8, o_r=8, o_h=8, n_kv=big, lk=1, **kw)
        assert lib.cs_cross_attention_workspace(C.byref(d), C.byref(n)) == B.CS_E_UNSUPPORTED and word in B.cs_last_error()
        assert attn(d) == B.CS_E_UNSUPPORTED
    d = attn_desc(n_kv=2 ** 20, lk=2 ** 20)
    assert lib.cs_kv4_attention_workspace(C.byref(d), C.byref(n)) == B.CS_E_UNSUPPORTED and n.value == 77


def test_scales_that_overflow():
    for s in (1e38, 3.4e38):
        assert attn(attn_desc(scale=s)) == B.CS_E_INVAL and "scale" in B.cs_last_error()


def test_the_workspace_holds_no_more_contexts_than_sets():
    """Over 4 bits, many bf16 rows read contexts that are unpacked first: as many as the sets that read
    them, not all of the cache."""
    n, one = C.c_size_t(0), C.c_size_t(0)
    big = dict(lq=300, heads_q=8, heads_kv=8, head_dim=128, lk=700)
    fn = B.lib().cs_kv4_attention_workspace
    assert fn(C.byref(attn_desc(n_q=1, n_kv=1, **big)), C.byref(one)) == B.CS_OK
    assert one.value >= 2 * 700 * 8 * 128 * 2
    for n_q, n_kv in ((1, 64), (3, 2000), (5, 5), (7, 2)):
        assert fn(C.byref(attn_desc(n_q=n_q, n_kv=n_kv, **big)), C.byref(n)) == B.CS_OK
        assert n.value <= min(n_q, n_kv) * one.value, (n_q, n_kv)


def test_many_rows_of_few_heads_share_a_long_context_out():
    """One key head of 1,032 rows over 131,072 keys makes nine blocks of 128 rows for 256 compute units:
    the keys are cut, as for fewer rows, which shows in the workspace."""
    n = C.c_size_t(0)
    few = dict(n_q=1, n_kv=1, lq=129, heads_q=8, heads_kv=1, head_dim=128)
    row = 128 * 4 + 8          # of a part: outputs, maximum and sum
    for dtype, fn, kv in ((B.CS_BF16, B.lib().cs_cross_attention_workspace, 0),
                          (B.CS_BF16, B.lib().cs_kv4_attention_workspace, 4 * 131072 * 128),
                          (B.CS_FP32, B.lib().cs_kv4_attention_workspace, 0)):
        assert fn(C.byref(attn_desc(dtype=dtype, lk=131072, **few)), C.byref(n)) == B.CS_OK
        assert n.value >= kv + 1032 * row * (7 if dtype == B.CS_FP32 else 28)
    # enough heads, or few keys: none
    for kw in (dict(heads_q=16, heads_kv=16, lq=1032, lk=131072), dict(heads_q=8, heads_kv=1, lq=129, lk=2048)):
        d = attn_desc(n_q=1, n_kv=1, head_dim=128, **kw)
        assert B.lib().cs_cross_attention_workspace(C.byref(d), C.byref(n)) == B.CS_OK and n.value == 0


@pytest.mark.parametrize("what", ["parts", "parts of a cache", "unpacked cache", "both"])
def test_every_workspace_that_is_needed_is_checked(what):
    n = C.c_size_t(0)
    if what == "parts":
        d, fn = attn_desc(lq=1, lk=1 << 20, k_b=1 << 28, v_b=1 << 28), B.lib().cs_cross_attention_workspace
        call = attn
    else:
        lq, lk = {"parts of a cache": (1, 1 << 20), "unpacked cache": (100, 600), "both": (100, 5000)}[what]
        d, fn = attn_desc(lq=lq, lk=lk), B.lib().cs_kv4_attention_workspace
        call = lambda d, **kw: kv4(d, cache(cap=lk), **kw)
    assert fn(C.byref(d), C.byref(n)) == B.CS_OK and n.value > 0
    for kw in (dict(), dict(work=P, nbytes=n.value - 1), dict(work=P + 8, nbytes=n.value), dict(nbytes=n.value)):
        assert call(d, **kw) == B.CS_E_INVAL and "workspace" in B.cs_last_error()
