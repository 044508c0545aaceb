"""The transformer with its projections in 8 bits (cs_model_init_proj) against the float64 oracle, as it is
and with its projections' weights and inputs rounded to 8 bits."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import dit as odit
from paper_2607_23159_amd import binding as B
from paper_2607_23159_amd import synth
from paper_2607_23159_amd.search import GpuModel, run_rollout
from parity import rel_l2, token_errors

PROJECTIONS = ("qkv_w", "o_w", "caq_w", "cao_w", "ffn1_w", "ffn2_w")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def rounded(x):
    """Rows of x as their 8-bit codes stand for them."""
    s = (np.abs(x).max(-1, keepdims=True) / 127).astype(np.float32).astype(np.float64)
    return np.round(x / np.where(s > 0, s, 1.0)) * s


def made(name, norm=B.CS_QK_NORM_FULL, init="stress"):
    m = synth.MODELS[name].with_dtype(synth.DTYPE_BF16)
    flat = synth.make_weights(m, init=init)
    W = {k: v.astype(np.float64) for k, v in synth.unflatten(m, flat).items()}
    return m, GpuModel(m, flat, qk_norm=norm, proj=B.CS_PROJ_8BIT), W


def run(gm, x, t, ctx):
    v = gm.velocity(torch.from_numpy(x.reshape(x.shape[0], -1)).cuda(), t, torch.from_numpy(ctx).cuda())
    return v.cpu().numpy().reshape(x.shape)


# A row's largest of up to 1536 values is at most some 5 of its deviations, so a code is off by
# 5 / 127 / sqrt(12) = 1.14e-2 of them in the mean square.  Two blocks round 12 weights and 12 inputs, each
# of at most the whole velocity's share: sqrt(24) x 1.14e-2 = 5.6e-2 from the oracle as it is, and 5.6e-3 of
# bf16.  From the oracle that rounds to 8 bits too, the inputs' codes differ by one where the 5.6e-3 that
# bf16 leaves them off passes a border: in the mean square sqrt(5 / 127 x 0.8 x 5.6e-3) = 1.33e-2 of
# the deviations at most, times sqrt(12) = 4.6e-2.
FAR, NEAR = 6.2e-2, 5.2e-2


@pytest.mark.parametrize("name,norm", [("tiny", B.CS_QK_NORM_FULL), ("tiny", B.CS_QK_NORM_HEAD), ("ragged", B.CS_QK_NORM_FULL),
                                       ("wan_mid", B.CS_QK_NORM_FULL)])
def test_velocity(name, norm, monkeypatch):
    m, gm, W = made(name, norm)
    ctx = synth.make_context(m, 31)
    n = 1 if name == "wan_mid" else 3
    x = synth.make_noise(m, n, seed0=900)
    v = run(gm, x, 0.6, ctx)
    eight = {id(w) for k, w in W.items() if k.endswith(PROJECTIONS) and not k.endswith(("cak_w", "cav_w"))}
    emb = odit.text_embedding(ctx, W)
    plain = odit.linear
    heads = norm == B.CS_QK_NORM_HEAD
    for i in range(n):
        ref = odit.velocity(x[i], 0.6, emb, W, m, head_norm=heads)
        with monkeypatch.context() as p:
            p.setattr(odit, "linear", lambda u, w, b: plain(rounded(u), rounded(w), b) if id(w) in eight else plain(u, w, b))
            ref8 = odit.velocity(x[i], 0.6, emb, W, m, head_norm=heads)
        assert rel_l2(ref8, ref) > 1e-3, "no projection was rounded"
        assert rel_l2(v[i], ref8) < NEAR and rel_l2(v[i], ref) < FAR, (rel_l2(v[i], ref8), rel_l2(v[i], ref))
    # one by one: bitwise the same
    for i in range(n if n > 1 else 0):
        assert np.array_equal(run(gm, x[i:i + 1], 0.6, ctx)[0], v[i])
    gm.close()


def test_few_tokens():
    """Latents of four tokens: the few-row product under every epilogue of the transformer."""
    m = dataclasses.replace(synth.MODELS["tiny"], lat_f=1, lat_h=4, lat_w=4, dtype=synth.DTYPE_BF16)
    flat = synth.make_weights(m, init="stress")
    W = {k: v.astype(np.float64) for k, v in synth.unflatten(m, flat).items()}
    gm = GpuModel(m, flat, proj=B.CS_PROJ_8BIT)
    ctx = synth.make_context(m, 33)
    x = synth.make_noise(m, 5, seed0=920)
    v = run(gm, x, 0.7, ctx)
    emb = odit.text_embedding(ctx, W)
    for i in range(5):       # five latents take other kernels than one
        assert np.array_equal(run(gm, x[i:i + 1], 0.7, ctx)[0], v[i])
        assert rel_l2(v[i], odit.velocity(x[i], 0.7, emb, W, m)) < FAR
    gm.close()


@pytest.mark.parametrize("name,frames", [("wan13b", 5), ("wan14b", 2)])
def test_many_tokens(name, frames):
    """The large tiles under every epilogue (v transposed, gated residual, GELU): a latent alone, whose products
    take other tiles, is bitwise what it is among others, and the compute type's result is near.  A token's
    error is held against the tokens' mean norm: twice the bound, as a token is up to twice that norm."""
    m = dataclasses.replace(synth.MODELS[name], n_blocks=1, lat_f=frames, dtype=synth.DTYPE_BF16)
    flat = synth.make_weights(m, init="stress")
    ctx = synth.make_context(m, 34)
    x = synth.make_noise(m, 3, seed0=930)
    gm = GpuModel(m, flat, proj=B.CS_PROJ_8BIT)
    v = run(gm, x, 0.4, ctx)
    for i in (0, 2):
        assert np.array_equal(run(gm, x[i:i + 1], 0.4, ctx)[0], v[i])
    gm.close()
    native = GpuModel(m, flat)
    ref = run(native, x, 0.4, ctx)
    native.close()
    for i in range(3):
        assert rel_l2(v[i], ref[i]) < FAR and token_errors(v[i], ref[i]).max() < 2 * FAR


def test_prompts_and_one_text_agree():
    m, gm, W = made("ragged")
    ctx = synth.make_context(m, 32)
    x = synth.make_noise(m, 2, seed0=910)
    a = run(gm, x, 0.3, ctx)
    ps = gm.prompts(torch.from_numpy(ctx[None]).cuda())
    b = ps.velocity(torch.from_numpy(x.reshape(2, -1)).cuda(), 0.3, [0, 0]).cpu().numpy().reshape(x.shape)
    assert rel_l2(a, b) < NEAR       # another attention kernel's bf16 roundings, through codes
    gm.close()


def test_rollouts():
    """No reuse at tau 0 and at range 1, and a seed alone as among others: bitwise."""
    wl = synth.make_workload("tiny", n_branch=2, init="stress", dtype=synth.DTYPE_BF16, n_cand=3)
    gm = GpuModel(wl.model, wl.weights, proj=B.CS_PROJ_8BIT)
    off = run_rollout(gm, wl, mode=synth.CACHE_OFF)
    zero = run_rollout(gm, wl, mode=synth.CACHE_ADAPTIVE, tau=0.0)
    pab = run_rollout(gm, wl, mode=synth.CACHE_PAB, pab_self=1, pab_cross=1)
    assert np.array_equal(off.latents, zero.latents) and np.array_equal(off.latents, pab.latents)
    reuse = run_rollout(gm, wl, mode=synth.CACHE_PAB, pab_self=2, pab_cross=3)
    assert np.isfinite(reuse.latents).all() and not np.array_equal(reuse.latents, off.latents)
    native = GpuModel(wl.model, wl.weights)
    ref = run_rollout(native, wl, mode=synth.CACHE_OFF)
    assert 1e-5 < rel_l2(off.latents, ref.latents) < FAR
    gm.close()
    native.close()
