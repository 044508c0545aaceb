"""Thin ctypes binding of ``libcachedsearch.so`` (the C ABI in include/cs.h).

Functions keep the C names and only marshal arguments: device buffers are
passed as integers or as objects with ``data_ptr()`` (torch tensors), HIP
streams as integers or objects with ``cuda_stream``.  Every non-OK status
raises :class:`CsError` carrying the library's message.  There is no
fallback: if the library is not built, importing anything that calls it
fails loudly.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Optional, Sequence, Tuple

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcachedsearch.so")

CS_OK, CS_E_INVAL, CS_E_NOMEM, CS_E_DEVICE, CS_E_STATE, CS_E_UNSUPPORTED = range(6)
CS_BF16, CS_FP32, CS_I8 = 0, 1, 2
CS_CACHE_OFF, CS_CACHE_ADAPTIVE, CS_CACHE_STATIC, CS_CACHE_PAB = 0, 1, 2, 3
CS_QK_NORM_FULL, CS_QK_NORM_HEAD = 0, 1
CS_KV_NATIVE, CS_KV_4BIT = 0, 1
CS_PROJ_NATIVE, CS_PROJ_8BIT = 0, 1
CS_ROPE_PAIRS, CS_ROPE_HALVES = 0, 1
CS_ACT_NONE, CS_ACT_GELU = 0, 1
(CS_K_SELF_ATTN, CS_K_CROSS_ATTN, CS_K_GEMM, CS_K_NORM, CS_K_DECIDE, CS_K_UPDATE, CS_K_SCORE,
 CS_K_OTHER) = range(8)
KERNEL_FAMILIES = ["self_attn", "cross_attn", "gemm", "norm", "decide", "update", "score", "other"]


class CsError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"cs status {status}: {msg}")
        self.status = status


class cs_model_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_blocks", "hidden", "heads", "head_dim", "ffn", "text_dim", "text_len", "freq_dim",
        "in_ch", "lat_f", "lat_h", "lat_w", "patch_t", "patch_h", "patch_w", "dtype")]


class cs_rollout_desc(C.Structure):
    _fields_ = [("n_cand", C.c_int32), ("n_steps", C.c_int32), ("n_branch", C.c_int32),
                ("k_warm", C.c_int32), ("k_cool", C.c_int32), ("static_k", C.c_int32),
                ("mode", C.c_int32), ("tau", C.c_float), ("guidance", C.c_float),
                ("timesteps", C.POINTER(C.c_float)),
                ("pab_self_range", C.c_int32), ("pab_cross_range", C.c_int32)]


class cs_rollout_stats_t(C.Structure):
    _fields_ = [("steps_done", C.c_int32), ("calls", C.c_int64), ("computed", C.c_int64),
                ("self_reused", C.c_int64), ("cross_reused", C.c_int64), ("n_cand", C.c_int32)]


class cs_qk_norm_desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "tokens", "heads_q", "heads_k", "head_dim", "rot_dim",
                                          "rope_rows", "rope_style")] + [("eps", C.c_float)] +
                [(n, C.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "qo_row", "qo_head", "ko_row",
                                          "ko_head", "q_gain_head", "k_gain_head")])


class cs_attn_desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "n_q", "n_kv", "lq", "lk", "heads_q", "heads_kv", "head_dim")] +
                [("scale", C.c_float)] +
                [(n, C.c_int64) for n in ("q_b", "q_r", "q_h", "k_b", "k_r", "k_h", "v_b", "v_r", "v_h", "o_b",
                                          "o_r", "o_h", "mask_b")])


class cs_kv4_cache(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")] +
                [(n, C.c_int32) for n in ("n_kv", "heads", "cap", "head_dim")])


class cs_kv4_rows(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "n_rows")] +
                [(n, C.c_int64) for n in ("k_row", "k_head", "v_row", "v_head")])


class cs_layer_norm_desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("x_dtype", "y_dtype", "groups", "rows", "dim", "unit_offset")] +
                [("eps", C.c_float)] + [(n, C.c_int64) for n in ("x_row", "y_row", "w_group", "b_group")])


class cs_layer_norm_grad_desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("x_dtype", "y_dtype", "groups", "rows", "dim", "unit_offset")] +
                [(n, C.c_int64) for n in ("x_row", "dy_row", "dx_row", "w_group", "dw_group", "db_group")])


class cs_i8_rows(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("dtype", "rows", "dim")] + [(n, C.c_int64) for n in ("x_row", "q_row")])


class cs_i8_weight(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("n", C.c_int32), ("k", C.c_int32)]


class cs_matmul_i8_desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("out_dtype", "rows", "n", "k", "act")] +
                [(n, C.c_int64) for n in ("a_row", "o_row")])


_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run paper_2607_23159_amd.build.build()")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
    pf, pd, pu8, pi32 = C.c_void_p, C.POINTER(C.c_double), C.c_void_p, C.POINTER(C.c_int32)
    sig = {
        "cs_model_weight_count": (i32, [C.POINTER(cs_model_desc), C.POINTER(sz)]),
        "cs_model_init": (i32, [C.POINTER(cs_model_desc), pf, sz, vp, C.POINTER(vp)]),
        "cs_model_init_norm": (i32, [C.POINTER(cs_model_desc), i32, pf, sz, vp, C.POINTER(vp)]),
        "cs_model_init_proj": (i32, [C.POINTER(cs_model_desc), i32, i32, pf, sz, vp, C.POINTER(vp)]),
        "cs_model_free": (None, [vp]),
        "cs_context_init": (i32, [vp, pf, pi32, i32, i32, C.POINTER(vp)]),
        "cs_context_free": (None, [vp]),
        "cs_velocity_context": (i32, [vp, vp, pf, pi32, i32, f32, pf]),
        "cs_velocity": (i32, [vp, pf, i32, f32, pf, pf]),
        "cs_rollout_init": (i32, [vp, C.POINTER(cs_rollout_desc), pf, pf, pf, C.POINTER(vp)]),
        "cs_rollout_free": (None, [vp]),
        "cs_cache_decide": (i32, [vp, i32, pu8, pu8, pd]),
        "cs_denoise_step": (i32, [vp, i32]),
        "cs_score": (i32, [vp, pf, pd]),
        "cs_score_noalloc": (i32, [pf, pf, i32, i64, pf, vp]),
        "cs_rollout_latents": (i32, [vp, pf]),
        "cs_rollout_stats": (i32, [vp, C.POINTER(cs_rollout_stats_t)]),
        "cs_rollout_enable_preview": (i32, [vp, i32]),
        "cs_preview_score": (i32, [vp, pf, pd]),
        "cs_rollout_retain": (i32, [vp, pi32, i32]),
        "cs_rollout_export": (i32, [vp, vp, C.POINTER(sz)]),
        "cs_rollout_import": (i32, [vp, vp, sz]),
        "cs_rank": (i32, [pd, pd, i32, pi32, pi32, pd, pi32]),
        "cs_qk_norm_rope": (i32, [C.POINTER(cs_qk_norm_desc)] + [vp] * 9),
        "cs_cross_attention_workspace": (i32, [C.POINTER(cs_attn_desc), C.POINTER(sz)]),
        "cs_cross_attention": (i32, [C.POINTER(cs_attn_desc)] + [vp] * 8 + [sz, vp]),
        "cs_kv4_attention_workspace": (i32, [C.POINTER(cs_attn_desc), C.POINTER(sz)]),
        "cs_kv4_attention": (i32, [C.POINTER(cs_attn_desc), vp, C.POINTER(cs_kv4_cache)] + [vp] * 5 + [sz, vp]),
        "cs_kv4_store": (i32, [C.POINTER(cs_kv4_cache), C.POINTER(cs_kv4_rows)] + [vp] * 4),
        "cs_kv4_load": (i32, [C.POINTER(cs_kv4_cache), C.POINTER(cs_kv4_rows)] + [vp] * 4),
        "cs_layer_norm": (i32, [C.POINTER(cs_layer_norm_desc)] + [vp] * 8),
        "cs_layer_norm_backward_workspace": (i32, [C.POINTER(cs_layer_norm_grad_desc), C.POINTER(sz)]),
        "cs_layer_norm_backward": (i32, [C.POINTER(cs_layer_norm_grad_desc)] + [vp] * 9 + [sz, vp]),
        "cs_i8_quantise": (i32, [C.POINTER(cs_i8_rows)] + [vp] * 4),
        "cs_i8_dequantise": (i32, [C.POINTER(cs_i8_rows)] + [vp] * 4),
        "cs_i8_weight_bytes": (i32, [i32, i32, C.POINTER(sz)]),
        "cs_i8_weight_pack": (i32, [C.POINTER(cs_i8_weight), i32, vp, i64, vp, vp]),
        "cs_matmul_i8_workspace": (i32, [C.POINTER(cs_matmul_i8_desc), C.POINTER(sz)]),
        "cs_matmul_i8": (i32, [C.POINTER(cs_matmul_i8_desc), vp, vp, C.POINTER(cs_i8_weight)] + [vp] * 3 + [sz, vp]),
        "cs_profile_enable": (i32, [vp, i32]),
        "cs_profile_reset": (i32, [vp]),
        "cs_profile_read": (i32, [vp, i32, pd, C.POINTER(i64)]),
        "cs_last_error": (C.c_char_p, []),
        "cs_debug_set_alloc_cap": (None, [sz]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(status: int) -> None:
    if status != CS_OK:
        raise CsError(status, lib().cs_last_error().decode(errors="replace"))


def _ptr(x, numel: Optional[int] = None, dtype: str = "float32", name: str = "buffer") -> Optional[int]:
    """Device address of ``x``: None, a raw integer address (passed through
    unchecked), or a tensor, which must be a contiguous device tensor of the
    given dtype holding at least ``numel`` elements."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not getattr(x, "is_cuda", False):
        raise ValueError(f"{name}: a device tensor is required (got {getattr(x, 'device', type(x))})")
    if str(x.dtype).rsplit(".", 1)[-1] != dtype:
        raise ValueError(f"{name}: dtype {x.dtype}, {dtype} required")
    if not x.is_contiguous():
        raise ValueError(f"{name}: tensor must be contiguous")
    if numel is not None and x.numel() < numel:
        raise ValueError(f"{name}: {x.numel()} elements, {numel} required")
    return int(x.data_ptr())


# Latent size D of every live model handle and the model of every live
# rollout handle, so that tensor arguments can be checked against the sizes
# the library will read or write.
_model_D = {}
_model_text = {}
_rollout_model = {}


def _latent_numel(model: int) -> Optional[int]:
    return _model_D.get(model)


def _stream(s) -> Optional[int]:
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return int(s.cuda_stream)


# ------------------------------------------------------------ descriptors
def model_desc(cfg, dtype: Optional[int] = None) -> cs_model_desc:
    """cs_model_desc from any object with the ModelCfg fields."""
    return cs_model_desc(cfg.n_blocks, cfg.hidden, cfg.heads, cfg.head_dim, cfg.ffn, cfg.text_dim,
                         cfg.text_len, cfg.freq_dim, cfg.in_ch, cfg.lat_f, cfg.lat_h, cfg.lat_w,
                         cfg.patch_t, cfg.patch_h, cfg.patch_w,
                         cfg.dtype if dtype is None else dtype)


class RolloutDesc:
    """cs_rollout_desc plus the timestep array it points to."""

    def __init__(self, roll, timesteps: Sequence[float], **override):
        kw = dict(n_cand=roll.n_cand, n_steps=roll.n_steps, n_branch=roll.n_branch,
                  k_warm=roll.k_warm, k_cool=roll.k_cool, static_k=roll.static_k,
                  mode=roll.mode, tau=roll.tau, guidance=roll.guidance,
                  pab_self=getattr(roll, "pab_self", 2), pab_cross=getattr(roll, "pab_cross", 6))
        kw.update(override)
        self.t = np.ascontiguousarray(np.asarray(timesteps, dtype=np.float32))
        self.c = cs_rollout_desc(kw["n_cand"], kw["n_steps"], kw["n_branch"], kw["k_warm"],
                                 kw["k_cool"], kw["static_k"], kw["mode"],
                                 float(kw["tau"]), float(kw["guidance"]),
                                 self.t.ctypes.data_as(C.POINTER(C.c_float)),
                                 int(kw["pab_self"]), int(kw["pab_cross"]))


# ------------------------------------------------------------------- calls
def cs_model_weight_count(desc: cs_model_desc) -> int:
    n = C.c_size_t(0)
    _check(lib().cs_model_weight_count(C.byref(desc), C.byref(n)))
    return n.value


def cs_model_init(desc: cs_model_desc, weights, n_weights: int, stream=None) -> int:
    return cs_model_init_norm(desc, CS_QK_NORM_FULL, weights, n_weights, stream)


def _opened(model, desc: cs_model_desc) -> int:
    _model_D[model.value] = desc.in_ch * desc.lat_f * desc.lat_h * desc.lat_w
    _model_text[model.value] = (desc.text_len, desc.text_dim)
    return model.value


def cs_model_init_norm(desc: cs_model_desc, qk_norm: int, weights, n_weights: int, stream=None) -> int:
    out = C.c_void_p()
    _check(lib().cs_model_init_norm(C.byref(desc), int(qk_norm), _ptr(weights, n_weights, name="weights"), n_weights,
                                    _stream(stream), C.byref(out)))
    return _opened(out, desc)


def cs_model_init_proj(desc: cs_model_desc, qk_norm: int, proj: int, weights, n_weights: int, stream=None) -> int:
    out = C.c_void_p()
    _check(lib().cs_model_init_proj(C.byref(desc), int(qk_norm), int(proj), _ptr(weights, n_weights, name="weights"),
                                    n_weights, _stream(stream), C.byref(out)))
    return _opened(out, desc)


def cs_model_free(model: int) -> None:
    lib().cs_model_free(model)
    _model_D.pop(model, None)
    _model_text.pop(model, None)


def cs_context_init(model: int, ctx, n_prompts: int, lens: Optional[Sequence[int]] = None,
                    kv_format: int = CS_KV_NATIVE) -> int:
    """Context handle of ``n_prompts`` prompts ``ctx`` [n_prompts][text_len][text_dim]; ``lens``: rows of each."""
    out = C.c_void_p()
    rows = _model_text.get(model)
    ln = None if lens is None else np.ascontiguousarray(np.asarray(lens, dtype=np.int32))
    if ln is not None and ln.size != n_prompts:
        raise ValueError(f"{ln.size} lengths for {n_prompts} prompts")
    _check(lib().cs_context_init(model, _ptr(ctx, None if rows is None else n_prompts * rows[0] * rows[1], name="ctx"),
                                 None if ln is None else ln.ctypes.data_as(C.POINTER(C.c_int32)), int(n_prompts),
                                 int(kv_format), C.byref(out)))
    return out.value


def cs_context_free(context: int) -> None:
    lib().cs_context_free(context)


def cs_velocity_context(model: int, context: int, x, n: int, t: float, v, prompt: Optional[Sequence[int]] = None) -> None:
    D = _latent_numel(model)
    nD = None if D is None else n * D
    of = None if prompt is None else np.ascontiguousarray(np.asarray(prompt, dtype=np.int32))
    if of is not None and of.size != n:
        raise ValueError(f"{of.size} prompts for {n} latents")
    _check(lib().cs_velocity_context(model, context, _ptr(x, nD, name="x"),
                                     None if of is None else of.ctypes.data_as(C.POINTER(C.c_int32)), n, float(t),
                                     _ptr(v, nD, name="v")))


def cs_velocity(model: int, x, n: int, t: float, ctx, v) -> None:
    D = _latent_numel(model)
    nD = None if D is None else n * D
    _check(lib().cs_velocity(model, _ptr(x, nD, name="x"), n, float(t), _ptr(ctx, name="ctx"),
                             _ptr(v, nD, name="v")))


def cs_rollout_init(model: int, desc: RolloutDesc, x1, ctx_cond, ctx_uncond=None) -> int:
    out = C.c_void_p()
    D = _latent_numel(model)
    _check(lib().cs_rollout_init(model, C.byref(desc.c),
                                 _ptr(x1, None if D is None else desc.c.n_cand * D, name="x1"),
                                 _ptr(ctx_cond, name="ctx_cond"), _ptr(ctx_uncond, name="ctx_uncond"),
                                 C.byref(out)))
    _rollout_model[out.value] = model
    return out.value


def cs_rollout_free(r: int) -> None:
    lib().cs_rollout_free(r)
    _rollout_model.pop(r, None)


def _rollout_D(r: int) -> Optional[int]:
    return _latent_numel(_rollout_model.get(r, 0))


def cs_cache_decide(r: int, step: int, n_streams: int, override_mask: Optional[np.ndarray] = None,
                    want: bool = True) -> Tuple[Optional[np.ndarray], Optional[np.ndarray]]:
    """Returns (mask [n_streams] uint8, a [n_streams] float64) when ``want``."""
    ovr = None
    if override_mask is not None:
        ovr = np.ascontiguousarray(np.asarray(override_mask, dtype=np.uint8).reshape(-1))
        assert ovr.size == n_streams
    mask = np.zeros(n_streams, np.uint8) if want else None
    a = np.zeros(n_streams, np.float64) if want else None
    _check(lib().cs_cache_decide(
        r, step, None if ovr is None else ovr.ctypes.data, None if mask is None else mask.ctypes.data,
        None if a is None else a.ctypes.data_as(C.POINTER(C.c_double))))
    return mask, a


def cs_denoise_step(r: int, step: int) -> None:
    _check(lib().cs_denoise_step(r, step))


def _current_n_cand(r: int, n_cand: int) -> None:
    cur = cs_rollout_stats(r).n_cand
    if n_cand != cur:
        raise ValueError(f"n_cand {n_cand} does not match the rollout's current {cur} candidates")


def cs_score(r: int, w, n_cand: int) -> np.ndarray:
    _current_n_cand(r, n_cand)
    out = np.zeros(n_cand, np.float64)
    _check(lib().cs_score(r, _ptr(w, _rollout_D(r), name="w"), out.ctypes.data_as(C.POINTER(C.c_double))))
    return out


def cs_score_noalloc(x, w, n: int, D: int, scores, stream=None) -> None:
    """Enqueue the scores of n latents x [n][D] into the device float64
    tensor ``scores`` [n]; allocates nothing and does not synchronise."""
    _check(lib().cs_score_noalloc(_ptr(x, n * D, name="x"), _ptr(w, D, name="w"), int(n), int(D),
                                  _ptr(scores, n, dtype="float64", name="scores"), _stream(stream)))


def cs_rollout_latents(r: int, dst) -> None:
    D = _rollout_D(r)
    n = cs_rollout_stats(r).n_cand
    _check(lib().cs_rollout_latents(r, _ptr(dst, None if D is None else n * D, name="dst")))


def cs_rollout_enable_preview(r: int, on: bool = True) -> None:
    _check(lib().cs_rollout_enable_preview(r, 1 if on else 0))


def cs_preview_score(r: int, w, n_cand: int) -> np.ndarray:
    _current_n_cand(r, n_cand)
    out = np.zeros(n_cand, np.float64)
    _check(lib().cs_preview_score(r, _ptr(w, _rollout_D(r), name="w"),
                                  out.ctypes.data_as(C.POINTER(C.c_double))))
    return out


def cs_rollout_retain(r: int, keep: Sequence[int]) -> None:
    k = np.ascontiguousarray(np.asarray(keep, dtype=np.int32))
    _check(lib().cs_rollout_retain(r, k.ctypes.data_as(C.POINTER(C.c_int32)), int(k.size)))


def cs_rollout_stats(r: int) -> cs_rollout_stats_t:
    s = cs_rollout_stats_t()
    _check(lib().cs_rollout_stats(r, C.byref(s)))
    return s


def cs_rollout_export(r: int) -> bytes:
    n = C.c_size_t(0)
    _check(lib().cs_rollout_export(r, None, C.byref(n)))
    buf = C.create_string_buffer(n.value)
    _check(lib().cs_rollout_export(r, buf, C.byref(n)))
    return buf.raw[:n.value]


def cs_rollout_import(r: int, data: bytes) -> None:
    buf = C.create_string_buffer(data, len(data))
    _check(lib().cs_rollout_import(r, buf, len(data)))


def cs_rank(s_cached: Sequence[float], s_full: Optional[Sequence[float]]):
    """(order_cached, order_full, rho, top1_agree); with ``s_full`` None only
    the order of ``s_cached`` is computed (the rest is None)."""
    a = np.ascontiguousarray(np.asarray(s_cached, np.float64))
    n = a.size
    oc = np.zeros(n, np.int32)
    pd = C.POINTER(C.c_double)
    pi = C.POINTER(C.c_int32)
    if s_full is None:
        _check(lib().cs_rank(a.ctypes.data_as(pd), None, n, oc.ctypes.data_as(pi), None, None, None))
        return oc.tolist(), None, None, None
    b = np.ascontiguousarray(np.asarray(s_full, np.float64))
    if b.size != n:
        raise ValueError(f"score vectors of different lengths {n} and {b.size}")
    of = np.zeros(n, np.int32)
    rho = C.c_double(0.0)
    top1 = C.c_int32(0)
    _check(lib().cs_rank(a.ctypes.data_as(pd), b.ctypes.data_as(pd), n, oc.ctypes.data_as(pi),
                         of.ctypes.data_as(pi), C.byref(rho), C.byref(top1)))
    return oc.tolist(), of.tolist(), rho.value, top1.value


# --------------------------------------------------------------- operators
# Descriptors are made once from tensors and kept; a call then takes tensors of
# the same shape, strides, type and device (or raw addresses, unchecked).  Tensors
# must be on the current device.  stream: a torch stream or a raw handle; None is
# torch's current stream, so that calls follow what torch enqueued before them and can
# be captured by torch.cuda.graph.
_DTYPES = {"bfloat16": CS_BF16, "float32": CS_FP32}


def _sig(x):
    return x.dtype, x.shape, x.stride(), x.device


def _same(x, sig, name: str) -> Optional[int]:
    """Address of a tensor that looks like the one its descriptor was made from."""
    if x is None or isinstance(x, int):
        return x
    if (x.dtype, x.shape, x.stride(), x.device) != sig:
        raise ValueError(f"{name}: the descriptor is for {sig}, got {_sig(x)}")
    return x.data_ptr()


def _on_current(device) -> None:
    import torch
    if device.index != torch.cuda.current_device():
        raise ValueError(f"tensors are on {device}, the current device is cuda:{torch.cuda.current_device()}")


def _op_stream(s, device) -> Optional[int]:
    if s is not None:
        return _stream(s)
    import torch
    # the call behind torch.cuda.current_stream(device).cuda_stream, without its objects
    return torch._C._cuda_getCurrentRawStream(device.index)


def _aux(x, numel: int, dtype: str, name: str, device) -> Optional[int]:
    """Address of an index tensor, a mask or the like on the operator's device."""
    if x is not None and not isinstance(x, int) and x.device != device:
        raise ValueError(f"{name}: on {x.device}, the operator is on {device}")
    return _ptr(x, numel, dtype, name)


class _OpDesc:
    """A descriptor with the tensors' signatures it stands for."""

    def __init__(self, c, **sig):
        self.c, self.ref, self.sig = c, C.byref(c), sig
        self.device = next(s[3] for s in sig.values() if s is not None)


def _op_tensors(dtype: str, ndim: int, **tensors):
    """Signatures of device tensors of one type and rank whose last axis is contiguous."""
    out, device = {}, None
    for name, x in tensors.items():
        if x is None:
            out[name] = None
            continue
        if not getattr(x, "is_cuda", False):
            raise ValueError(f"{name}: a device tensor is required (got {getattr(x, 'device', type(x))})")
        if str(x.dtype).rsplit(".", 1)[-1] != dtype:
            raise ValueError(f"{name}: dtype {x.dtype}, {dtype} required")
        if x.dim() != ndim:
            raise ValueError(f"{name}: {x.dim()} axes, {ndim} required")
        if x.shape[-1] > 1 and x.stride(-1) != 1:
            raise ValueError(f"{name}: the last axis must be contiguous")
        if device is not None and x.device != device:
            raise ValueError(f"{name}: on {x.device}, the others on {device}")
        device = x.device
        out[name] = _sig(x)
    return out


def _float_dtype(x) -> str:
    d = str(x.dtype).rsplit(".", 1)[-1]
    if d not in _DTYPES:
        raise ValueError(f"dtype {x.dtype}, bfloat16 or float32 required")
    return d


def qk_norm_desc(q, k, q_out, k_out, q_gain, k_gain, rope=None, style: int = CS_ROPE_PAIRS,
                 eps: float = 1e-6) -> _OpDesc:
    """Descriptor of cs_qk_norm_rope.  q, q_out: [tokens][heads_q][head_dim]; k, k_out:
    [tokens][heads_k][head_dim]; gains [heads or 1][head_dim]; rope [rope_rows][rot_dim / 2][2] or
    None.  q with its output and gain, or k with its, may be None."""
    one = q if q is not None else k
    if one is None:
        raise ValueError("q and k are both None")
    t = _float_dtype(one)
    sig = _op_tensors(t, 3, q=q, k=k, q_out=q_out, k_out=k_out)
    sig.update(_op_tensors("float32", 2, q_gain=q_gain, k_gain=k_gain))
    sig.update(_op_tensors("float32", 3, rope=rope))
    tokens, dim = one.shape[0], one.shape[2]
    dims = {}
    for n, x, o, g in (("q", q, q_out, q_gain), ("k", k, k_out, k_gain)):
        if (x is None) != (o is None) or (x is None) != (g is None):
            raise ValueError(f"{n}, {n}_out and {n}_gain go together")
        if x is None:
            dims[n] = (0, 0, 0, 0, 0, 0)
            continue
        if x.shape[0] != tokens or x.shape[2] != dim or o.shape != x.shape:
            raise ValueError(f"{n}: shape {tuple(x.shape)}, output {tuple(o.shape)}, {tokens} tokens of {dim} channels")
        if g.shape[1] != dim or g.shape[0] not in (1, x.shape[1]):
            raise ValueError(f"{n}_gain: shape {tuple(g.shape)}")
        dims[n] = (x.shape[1], x.stride(0), x.stride(1), o.stride(0), o.stride(1), 0 if g.shape[0] == 1 else g.stride(0))
    rows, rot = 0, 0
    if rope is not None:
        if rope.shape[2] != 2 or not rope.is_contiguous():
            raise ValueError("rope: a contiguous [rows][rot_dim / 2][2] tensor is required")
        rows, rot = rope.shape[0], 2 * rope.shape[1]
    (hq, q0, q1, qo0, qo1, qg), (hk, k0, k1, ko0, ko1, kg) = dims["q"], dims["k"]
    return _OpDesc(cs_qk_norm_desc(_DTYPES[t], tokens, hq, hk, dim, rot, rows, style, eps, q0, q1, k0, k1, qo0, qo1,
                                   ko0, ko1, qg, kg), **sig)


def cs_qk_norm_rope(desc: _OpDesc, q, k, q_out, k_out, q_gain, k_gain, rope=None, pos=None, stream=None) -> None:
    """``pos``: int32 device tensor [tokens] or None."""
    _on_current(desc.device)
    s = desc.sig
    _check(lib().cs_qk_norm_rope(desc.ref, _same(q, s["q"], "q"), _same(k, s["k"], "k"),
                                 _same(q_out, s["q_out"], "q_out"), _same(k_out, s["k_out"], "k_out"),
                                 _same(q_gain, s["q_gain"], "q_gain"), _same(k_gain, s["k_gain"], "k_gain"),
                                 _same(rope, s["rope"], "rope"),
                                 _aux(pos, desc.c.tokens, "int32", "pos", desc.device),
                                 _op_stream(stream, desc.device)))


class Kv4Cache(_OpDesc):
    """A 4-bit cache over four contiguous uint8 device tensors: codes
    [n_kv][heads][cap][head_dim / 2] and scales [n_kv][heads][cap][head_dim / 32], of
    the keys and of the values.  Keeps the tensors."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        sig = _op_tensors("uint8", 4, k_codes=k_codes, k_scales=k_scales, v_codes=v_codes, v_scales=v_scales)
        n, h, cap, half = k_codes.shape
        for name, x in (("k_codes", k_codes), ("v_codes", v_codes), ("k_scales", k_scales), ("v_scales", v_scales)):
            want = (n, h, cap, half if name.endswith("codes") else half // 16)
            if tuple(x.shape) != want or not x.is_contiguous():
                raise ValueError(f"{name}: a contiguous {want} tensor is required, got {tuple(x.shape)}")
        self.tensors = (k_codes, k_scales, v_codes, v_scales)
        super().__init__(cs_kv4_cache(*(x.data_ptr() for x in self.tensors), n, h, cap, 2 * half), **sig)
        self._rows = {}

    def rows(self, k, v) -> _OpDesc:
        """cs_kv4_rows of tensors [n_rows][heads][head_dim] shaped like k and v (kept)."""
        key = (k.dtype, k.shape, k.stride(), k.device, v.dtype, v.shape, v.stride(), v.device)
        d = self._rows.get(key)
        if d is None:
            t = _float_dtype(k)
            sig = _op_tensors(t, 3, k=k, v=v)
            want = (k.shape[0], self.c.heads, self.c.head_dim)
            if tuple(k.shape) != want or tuple(v.shape) != want or k.device != self.device:
                raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)}: {want} on {self.device} required")
            d = _OpDesc(cs_kv4_rows(_DTYPES[t], want[0], k.stride(0), k.stride(1), v.stride(0), v.stride(1)), **sig)
            if len(self._rows) >= 64:   # layouts of a serving loop are few
                self._rows.clear()
            self._rows[key] = d
        return d


def cs_kv4_store(cache: Kv4Cache, k, v, slots=None, stream=None) -> None:
    """Rows k, v [n_rows][heads][head_dim] into the cache; ``slots``: int32 device tensor or None."""
    _on_current(cache.device)
    d = cache.rows(k, v)
    _check(lib().cs_kv4_store(cache.ref, d.ref, k.data_ptr(), v.data_ptr(), _aux(slots, d.c.n_rows, "int32", "slots", cache.device),
                              _op_stream(stream, cache.device)))


def cs_kv4_load(cache: Kv4Cache, k, v, slots=None, stream=None) -> None:
    """The values that rows of the cache stand for into k and v."""
    _on_current(cache.device)
    d = cache.rows(k, v)
    _check(lib().cs_kv4_load(cache.ref, d.ref, k.data_ptr(), v.data_ptr(), _aux(slots, d.c.n_rows, "int32", "slots", cache.device),
                             _op_stream(stream, cache.device)))


def _attn_desc(q, o, n_kv, lk, heads_kv, dim, kv_strides, scale, sig) -> _OpDesc:
    if o.shape != q.shape or q.shape[3] != dim:
        raise ValueError(f"q {tuple(q.shape)}, o {tuple(o.shape)}, {dim} channels")
    if scale is None:
        scale = 1.0 / math.sqrt(dim)
    n, lq, h, _ = q.shape
    return _OpDesc(cs_attn_desc(_DTYPES[_float_dtype(q)], n, n_kv, lq, lk, h, heads_kv, dim, scale, *q.stride()[:3],
                                *kv_strides, *o.stride()[:3], lk), **sig)


def attn_desc(q, k, v, o, scale: Optional[float] = None) -> _OpDesc:
    """Descriptor of cs_cross_attention.  q, o: [n_q][lq][heads_q][head_dim]; k, v:
    [n_kv][lk][heads_kv][head_dim].  scale: None for 1 / sqrt(head_dim)."""
    sig = _op_tensors(_float_dtype(q), 4, q=q, k=k, v=v, o=o)
    if v.shape != k.shape:
        raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} differ")
    n_kv, lk, hkv, dim = k.shape
    return _attn_desc(q, o, n_kv, lk, hkv, dim, (*k.stride()[:3], *v.stride()[:3]), scale, sig)


def kv4_attn_desc(q, cache: Kv4Cache, o, scale: Optional[float] = None) -> _OpDesc:
    """Descriptor of cs_kv4_attention over a cache."""
    sig = _op_tensors(_float_dtype(q), 4, q=q, o=o)
    if q.device != cache.device:
        raise ValueError(f"q on {q.device}, the cache on {cache.device}")
    c = cache.c
    return _attn_desc(q, o, c.n_kv, c.cap, c.heads, c.head_dim, (0,) * 6, scale, sig)


def cs_cross_attention_workspace(desc: _OpDesc) -> int:
    n = C.c_size_t(0)
    _check(lib().cs_cross_attention_workspace(desc.ref, C.byref(n)))
    return n.value


def cs_kv4_attention_workspace(desc: _OpDesc) -> int:
    n = C.c_size_t(0)
    _check(lib().cs_kv4_attention_workspace(desc.ref, C.byref(n)))
    return n.value


def _workspace(work, device):
    """Address and bytes of a workspace (any contiguous tensor, a raw address, or None)."""
    if work is None:
        return None, 0
    if isinstance(work, int):
        return work, 1 << 62    # unchecked
    if work.device != device or not work.is_contiguous():
        raise ValueError(f"work: a contiguous tensor on {device} is required")
    return work.data_ptr(), work.numel() * work.element_size()


def _attn_rest(desc: _OpDesc, kv_of, kv_len, kv_mask, work):
    """Addresses of the index tensors (int32), the mask ([n_kv][lk] uint8, contiguous) and the
    workspace, and the workspace's bytes."""
    c, dev = desc.c, desc.device
    work, nbytes = _workspace(work, dev)
    if kv_mask is not None and not isinstance(kv_mask, int) and kv_mask.dim() > 1 and kv_mask.shape[-1] != c.lk:
        raise ValueError(f"kv_mask: rows of {kv_mask.shape[-1]} keys, {c.lk} required")
    return (_aux(kv_of, c.n_q, "int32", "kv_of", dev), _aux(kv_len, c.n_kv, "int32", "kv_len", dev),
            _aux(kv_mask, c.n_kv * c.lk, "uint8", "kv_mask", dev), work, nbytes)


def cs_cross_attention(desc: _OpDesc, q, k, v, o, kv_of=None, kv_len=None, kv_mask=None, work=None,
                       stream=None) -> None:
    _on_current(desc.device)
    s = desc.sig
    of, ln, mask, w, nbytes = _attn_rest(desc, kv_of, kv_len, kv_mask, work)
    _check(lib().cs_cross_attention(desc.ref, _same(q, s["q"], "q"), _same(k, s["k"], "k"), _same(v, s["v"], "v"), of, ln,
                                    mask, _same(o, s["o"], "o"), w, nbytes, _op_stream(stream, desc.device)))


def cs_kv4_attention(desc: _OpDesc, q, cache: Kv4Cache, o, kv_of=None, kv_len=None, kv_mask=None, work=None,
                     stream=None) -> None:
    _on_current(desc.device)
    if cache.device != desc.device:
        raise ValueError(f"the cache is on {cache.device}, the descriptor's tensors on {desc.device}")
    s = desc.sig
    of, ln, mask, w, nbytes = _attn_rest(desc, kv_of, kv_len, kv_mask, work)
    _check(lib().cs_kv4_attention(desc.ref, _same(q, s["q"], "q"), cache.ref, of, ln, mask, _same(o, s["o"], "o"), w,
                                  nbytes, _op_stream(stream, desc.device)))


def _given(x, sig, name: str) -> Optional[int]:
    """_same for a tensor that is absent exactly where its descriptor was made without it."""
    if (x is None) != (sig is None):
        raise ValueError(f"{name}: the descriptor was made with{'out' if sig is None else ''} it")
    return _same(x, sig, name)


_float32 = None      # torch.float32, once torch is there


def _vector(x, n: int, name: str, device) -> Optional[int]:
    """Address of n fp32 values on the operator's device, or None."""
    global _float32
    if x is None or isinstance(x, int):
        return x
    if _float32 is None:
        import torch
        _float32 = torch.float32
    # what _aux checks, without making names of types (1 us)
    if x.dtype is _float32 and x.device == device and x.numel() >= n and x.is_contiguous():
        return x.data_ptr()
    return _aux(x, n, "float32", name, device)


def _params(dim: int, groups: int, **tensors):
    """Signatures of fp32 [groups][dim] tensors, and their strides from group to group."""
    sig = _op_tensors("float32", 2, **tensors)
    for n, x in tensors.items():
        if x is not None and tuple(x.shape) != (groups, dim):
            raise ValueError(f"{n}: shape {tuple(x.shape)}, {(groups, dim)} required")
    return sig, [0 if x is None else x.stride(0) for x in tensors.values()]


def _one_device(sig) -> None:
    devices = {s[3] for s in sig.values() if s is not None}
    if len(devices) > 1:
        raise ValueError(f"tensors on {sorted(map(str, devices))}")


def _norm_rows(x, groups: int):
    """Rows of a group and channels of x [groups * rows][dim]."""
    if groups < 1 or x.shape[0] % groups:
        raise ValueError(f"{x.shape[0]} rows are not {groups} groups")
    return x.shape[0] // groups, x.shape[1]


def layer_norm_desc(x, y, weight=None, bias=None, groups: int = 1, unit_offset: bool = False,
                    eps: float = 1e-6) -> _OpDesc:
    """Descriptor of cs_layer_norm.  x, y: [groups * rows][dim], y bfloat16, float32 or int8 (with a
    scale a row); weight, bias: [groups][dim] or None."""
    sig = _op_tensors(_float_dtype(x), 2, x=x)
    i8 = str(y.dtype).rsplit(".", 1)[-1] == "int8"
    sig.update(_op_tensors("int8" if i8 else _float_dtype(y), 2, y=y))
    rows, dim = _norm_rows(x, groups)
    if y.shape != x.shape:
        raise ValueError(f"x {tuple(x.shape)} and y {tuple(y.shape)} differ")
    p, strides = _params(dim, groups, weight=weight, bias=bias)
    sig.update(p)
    _one_device(sig)
    return _OpDesc(cs_layer_norm_desc(_DTYPES[_float_dtype(x)], CS_I8 if i8 else _DTYPES[_float_dtype(y)], groups, rows,
                                      dim, int(unit_offset), eps, x.stride(0), y.stride(0), *strides), **sig)


def cs_layer_norm(desc: _OpDesc, x, y, weight=None, bias=None, y_scale=None, mean=None, rstd=None, stream=None) -> None:
    """``y_scale``: float32 [rows in all], required where y is int8; ``mean``, ``rstd``: the same or None."""
    _on_current(desc.device)
    s, dev, n = desc.sig, desc.device, desc.c.groups * desc.c.rows
    _check(lib().cs_layer_norm(desc.ref, _same(x, s["x"], "x"), _given(weight, s["weight"], "weight"),
                               _given(bias, s["bias"], "bias"), _same(y, s["y"], "y"), _vector(y_scale, n, "y_scale", dev),
                               _vector(mean, n, "mean", dev), _vector(rstd, n, "rstd", dev), _op_stream(stream, dev)))


def layer_norm_grad_desc(x, dy, weight=None, dx=None, dweight=None, dbias=None, groups: int = 1,
                         unit_offset: bool = False) -> _OpDesc:
    """Descriptor of cs_layer_norm_backward.  x, dy, dx: [groups * rows][dim], dx of x's type or None;
    weight, dweight, dbias: float32 [groups][dim] or None."""
    sig = _op_tensors(_float_dtype(x), 2, x=x, dx=dx)
    sig.update(_op_tensors(_float_dtype(dy), 2, dy=dy))
    rows, dim = _norm_rows(x, groups)
    for n, t in (("dy", dy), ("dx", dx)):
        if t is not None and t.shape != x.shape:
            raise ValueError(f"x {tuple(x.shape)} and {n} {tuple(t.shape)} differ")
    p, strides = _params(dim, groups, weight=weight, dweight=dweight, dbias=dbias)
    sig.update(p)
    _one_device(sig)
    return _OpDesc(cs_layer_norm_grad_desc(_DTYPES[_float_dtype(x)], _DTYPES[_float_dtype(dy)], groups, rows, dim,
                                           int(unit_offset), x.stride(0), dy.stride(0), 0 if dx is None else dx.stride(0),
                                           *strides), **sig)


def cs_layer_norm_backward_workspace(desc: _OpDesc) -> int:
    n = C.c_size_t(0)
    _check(lib().cs_layer_norm_backward_workspace(desc.ref, C.byref(n)))
    return n.value


def cs_layer_norm_backward(desc: _OpDesc, x, dy, weight, mean, rstd, dx=None, dweight=None, dbias=None, work=None,
                           stream=None) -> None:
    """``mean``, ``rstd``: float32 [rows in all], as cs_layer_norm wrote them."""
    _on_current(desc.device)
    s, dev, n = desc.sig, desc.device, desc.c.groups * desc.c.rows
    work, nbytes = _workspace(work, dev)
    _check(lib().cs_layer_norm_backward(desc.ref, _same(x, s["x"], "x"), _same(dy, s["dy"], "dy"),
                                        _given(weight, s["weight"], "weight"), _vector(mean, n, "mean", dev),
                                        _vector(rstd, n, "rstd", dev), _given(dx, s["dx"], "dx"),
                                        _given(dweight, s["dweight"], "dweight"), _given(dbias, s["dbias"], "dbias"), work,
                                        nbytes, _op_stream(stream, dev)))


def i8_rows_desc(x, codes, scales) -> _OpDesc:
    """Descriptor of cs_i8_quantise and cs_i8_dequantise.  x, codes: [rows][dim], codes int8;
    scales: float32 [rows]."""
    t = _float_dtype(x)
    sig = _op_tensors(t, 2, x=x)
    sig.update(_op_tensors("int8", 2, codes=codes))
    sig.update(_op_tensors("float32", 1, scales=scales))
    if codes.shape != x.shape or scales.shape[0] != x.shape[0]:
        raise ValueError(f"x {tuple(x.shape)}, codes {tuple(codes.shape)}, scales {tuple(scales.shape)}")
    _one_device(sig)
    return _OpDesc(cs_i8_rows(_DTYPES[t], x.shape[0], x.shape[1], x.stride(0), codes.stride(0)), **sig)


def cs_i8_quantise(desc: _OpDesc, x, codes, scales, stream=None) -> None:
    _on_current(desc.device)
    s = desc.sig
    _check(lib().cs_i8_quantise(desc.ref, _same(x, s["x"], "x"), _same(codes, s["codes"], "codes"),
                                _same(scales, s["scales"], "scales"), _op_stream(stream, desc.device)))


def cs_i8_dequantise(desc: _OpDesc, codes, scales, x, stream=None) -> None:
    """The values that codes stand for into x."""
    _on_current(desc.device)
    s = desc.sig
    _check(lib().cs_i8_dequantise(desc.ref, _same(codes, s["codes"], "codes"), _same(scales, s["scales"], "scales"),
                                  _same(x, s["x"], "x"), _op_stream(stream, desc.device)))


def cs_i8_weight_bytes(n: int, k: int) -> int:
    out = C.c_size_t(0)
    _check(lib().cs_i8_weight_bytes(n, k, C.byref(out)))
    return out.value


class I8Weight(_OpDesc):
    """8-bit weights [n][k] in the layout of the products: an int8 tensor of cs_i8_weight_bytes
    codes and a float32 tensor of n scales, made here, to be filled by cs_i8_weight_pack."""

    def __init__(self, n: int, k: int, device="cuda"):
        import torch
        self.tensors = (torch.empty(cs_i8_weight_bytes(n, k), dtype=torch.int8, device=device),
                        torch.empty(n, dtype=torch.float32, device=device))
        codes, scales = self.tensors
        super().__init__(cs_i8_weight(codes.data_ptr(), scales.data_ptr(), n, k), codes=_sig(codes), scales=_sig(scales))


def cs_i8_weight_pack(weight: I8Weight, w, scales=None, stream=None) -> None:
    """w: [n][k] of bfloat16 or float32, or int8 codes with their ``scales`` (float32 [n])."""
    _on_current(weight.device)
    i8 = str(w.dtype).rsplit(".", 1)[-1] == "int8"
    sig = _op_tensors("int8" if i8 else _float_dtype(w), 2, w=w)
    c = weight.c
    if tuple(w.shape) != (c.n, c.k) or sig["w"][3] != weight.device:
        raise ValueError(f"w: shape {tuple(w.shape)} on {w.device}, {(c.n, c.k)} on {weight.device} required")
    _check(lib().cs_i8_weight_pack(weight.ref, CS_I8 if i8 else _DTYPES[_float_dtype(w)], w.data_ptr(), w.stride(0),
                                   _vector(scales, c.n, "scales", weight.device), _op_stream(stream, weight.device)))


def matmul_i8_desc(codes, scales, weight: I8Weight, out, act: int = CS_ACT_NONE) -> _OpDesc:
    """Descriptor of cs_matmul_i8.  codes: int8 [rows][k]; scales: float32 [rows]; out: [rows][n]."""
    t = _float_dtype(out)
    sig = _op_tensors("int8", 2, codes=codes)
    sig.update(_op_tensors("float32", 1, scales=scales))
    sig.update(_op_tensors(t, 2, out=out))
    c, rows = weight.c, codes.shape[0]
    if codes.shape[1] != c.k or scales.shape[0] != rows or tuple(out.shape) != (rows, c.n):
        raise ValueError(f"codes {tuple(codes.shape)}, scales {tuple(scales.shape)}, out {tuple(out.shape)}, weight {(c.n, c.k)}")
    sig["weight"] = weight.sig["codes"]
    _one_device(sig)
    return _OpDesc(cs_matmul_i8_desc(_DTYPES[t], rows, c.n, c.k, act, codes.stride(0), out.stride(0)), **sig)


def cs_matmul_i8_workspace(desc: _OpDesc) -> int:
    n = C.c_size_t(0)
    _check(lib().cs_matmul_i8_workspace(desc.ref, C.byref(n)))
    return n.value


def cs_matmul_i8(desc: _OpDesc, codes, scales, weight: I8Weight, out, bias=None, work=None, stream=None) -> None:
    """``bias``: float32 [n] or None."""
    _on_current(desc.device)
    if weight.device != desc.device:
        raise ValueError(f"the weight is on {weight.device}, the descriptor's tensors on {desc.device}")
    s, dev = desc.sig, desc.device
    work, nbytes = _workspace(work, dev)
    _check(lib().cs_matmul_i8(desc.ref, _same(codes, s["codes"], "codes"), _same(scales, s["scales"], "scales"), weight.ref,
                              _vector(bias, desc.c.n, "bias", dev), _same(out, s["out"], "out"), work, nbytes,
                              _op_stream(stream, dev)))


def cs_profile_enable(model: int, on: bool) -> None:
    _check(lib().cs_profile_enable(model, 1 if on else 0))


def cs_profile_reset(model: int) -> None:
    _check(lib().cs_profile_reset(model))


def cs_profile_read(model: int, family: int) -> Tuple[float, int]:
    ms = C.c_double(0.0)
    n = C.c_int64(0)
    _check(lib().cs_profile_read(model, family, C.byref(ms), C.byref(n)))
    return ms.value, n.value


def cs_last_error() -> str:
    return lib().cs_last_error().decode(errors="replace")
