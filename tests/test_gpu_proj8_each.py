"""Each of the transformer's projections in 8 bits by itself: one-block models in which the rounding of one
projection's weights, or of its inputs, is so coarse that a run that leaves it out is far off; and rollouts in 8
bits against the native ones."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import dit as odit
from paper_2607_23159_amd import binding as B
from paper_2607_23159_amd import synth
from paper_2607_23159_amd.search import GpuModel, run_rollout
from parity import check_ranking, rel_l2
from test_gpu_proj8 import FAR, PROJECTIONS, rounded, run


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


BRANCH = {"qkv_w": "o_w", "o_w": "o_w", "caq_w": "cao_w", "cao_w": "cao_w", "ffn1_w": "ffn2_w", "ffn2_w": "ffn2_w"}
# steps of two standard deviations: 254 of them in the one channel of a row that sets its scale
WIDE = 254.0
INPUT_STD = {"qkv_w": 1.0, "caq_w": 1.0, "ffn1_w": 1.0, "o_w": 0.3, "cao_w": 0.09, "ffn2_w": 0.32}


def coarse(m, name, side, c=5):
    """Weights of a one-block model whose velocity is the named projection's branch for the most part.  Channel c
    of the projection's input adds nothing, but sets the scales: of the weights, whose column c is
    large where the input is 0, or of the input, which is large where column c is 0."""
    flat = synth.make_weights(m, init="stress").copy()
    W = {k.split(".")[-1]: v for k, v in synth.unflatten(m, flat).items()}
    d = m.hidden
    for out in ("o_w", "cao_w", "ffn2_w"):
        W[out] *= 16.0 if out == BRANCH[name] else 0.0
    W["q_gain"] *= 3.0
    W["caq_gain"] *= 3.0
    if side == "weights":
        W[name][:, c] = WIDE * W[name].std()
        value = 0.0
    else:
        W[name][:, c] = 0.0
        value = WIDE * INPUT_STD[name]
    if name in ("qkv_w", "ffn1_w"):      # a shift of `value` and a gain of 0 at every time
        for row, v in ((0 if name == "qkv_w" else 3, value), (1 if name == "qkv_w" else 4, -1.0)):
            W["mod_w"][row * d + c] = 0.0
            W["mod_b"][row * d + c] = 0.0
            W["mod"].reshape(6, d)[row, c] = v
    elif name == "caq_w":
        W["ca_ln_g"][c], W["ca_ln_b"][c] = 0.0, value
    else:                                # a value, or a hidden unit, of `value` for every token
        src, row = {"o_w": ("qkv", 2 * d + c), "cao_w": ("cav", c), "ffn2_w": ("ffn1", c)}[name]
        W[src + "_w"][row], W[src + "_b"][row] = 0.0, value
    return flat


# Simulated on the host, with the oracle rounding to bf16 where the run does: its distance from the oracle that
# rounds to 8 bits is 1.0 to 1.9e-2 with coarse weights, and 4.2 to 14e-2 with coarse inputs, where a
# value that bf16 leaves off by 1e-2 moves by a step of 2 deviations wherever it passes a border.  Twice that.
TOLERANCE = {"weights": 4e-2, "inputs": 0.28}


@pytest.mark.parametrize("side", ["weights", "inputs"])
@pytest.mark.parametrize("name", PROJECTIONS)
def test_each_projection_is_rounded(name, side, monkeypatch):
    m = dataclasses.replace(synth.MODELS["tiny"], n_blocks=1, dtype=synth.DTYPE_BF16)
    flat = coarse(m, name, side)
    W = {k: v.astype(np.float64) for k, v in synth.unflatten(m, flat).items()}
    eight = {id(w): k.split(".")[-1] for k, w in W.items() if k.split(".")[-1] in PROJECTIONS}
    ctx, x = synth.make_context(m, 31), synth.make_noise(m, 2, seed0=940)
    emb, plain = odit.text_embedding(ctx, W), odit.linear

    def oracle(xi, without=None):
        with monkeypatch.context() as p:
            p.setattr(odit, "linear", lambda u, w, b: plain(u, w, b) if eight.get(id(w), without) == without
                      else plain(rounded(u), rounded(w), b))
            return odit.velocity(xi, 0.6, emb, W, m)
    gm = GpuModel(m, flat, proj=B.CS_PROJ_8BIT)
    v = run(gm, x, 0.6, ctx)
    gm.close()
    for i in range(2):
        ref, left_out = oracle(x[i]), oracle(x[i], name)
        assert rel_l2(left_out, ref) > 1.2 * TOLERANCE[side], "the case does not tell"
        print(name, side, "off %.4f, left out %.3f" % (rel_l2(v[i], ref), rel_l2(left_out, ref)), flush=True)
        assert rel_l2(v[i], ref) < TOLERANCE[side]
        assert rel_l2(v[i], ref) < 0.5 * rel_l2(v[i], left_out)


@pytest.mark.parametrize("mode", [synth.CACHE_OFF, synth.CACHE_ADAPTIVE, synth.CACHE_STATIC, synth.CACHE_PAB])
def test_a_seed_alone_is_what_it_is_among_others(mode):
    wl = synth.make_workload("tiny", n_branch=2, init="stress", dtype=synth.DTYPE_BF16, n_cand=3)
    gm = GpuModel(wl.model, wl.weights, proj=B.CS_PROJ_8BIT)
    among = run_rollout(gm, wl, mode=mode)
    alone = run_rollout(gm, wl, mode=mode, n_cand=1)
    gm.close()
    assert np.array_equal(alone.latents[0], among.latents[0]) and alone.scores[0] == among.scores[0]
    assert np.array_equal(alone.masks, among.masks[:, :2])


@pytest.mark.parametrize("tau", [0.05, 0.1, 0.2])
def test_skip_schedules_are_those_of_the_compute_type(tau):
    """Native and 8-bit rollouts decide alike but where an indicator is near tau: an indicator is a relative change of
    what the velocities move, so that velocities off by FAR move it by at most 2 FAR of itself."""
    wl = synth.make_workload("tiny", init="paper", dtype=synth.DTYPE_BF16, n_cand=4)
    runs = []
    for proj in (B.CS_PROJ_8BIT, B.CS_PROJ_NATIVE):
        gm = GpuModel(wl.model, wl.weights, proj=proj)
        runs.append(run_rollout(gm, wl, mode=synth.CACHE_ADAPTIVE, tau=tau))
        gm.close()
    eight, native = runs
    same = 0
    for s in range(native.masks.shape[1]):
        for k in range(native.masks.shape[0]):
            if eight.masks[k, s] != native.masks[k, s]:
                assert abs(native.a[k, s] - tau) <= 2 * FAR * tau, (s, k, native.a[k, s])
                break
        else:
            same += 1
            assert rel_l2(eight.latents[s], native.latents[s]) < FAR
    print("streams with one schedule:", same, "computed", eight.computed, native.computed, flush=True)


@pytest.mark.parametrize("proj", [B.CS_PROJ_NATIVE, B.CS_PROJ_8BIT])
def test_more_tokens_than_a_launch_has_rows(proj):
    """2^24 tokens with a feed-forward wider than 2048: a workgroup a row would pass a launch's 2^32 work items.  A
    latent is bitwise what it is alone."""
    m = dataclasses.replace(synth.MODELS["tiny"], n_blocks=1, hidden=64, heads=2, ffn=2112, lat_f=1, lat_h=128, lat_w=128,
                            dtype=synth.DTYPE_BF16)
    n = 4096
    assert n * m.tokens == 1 << 24
    x = torch.randn(n, m.latent_numel, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    ctx = torch.from_numpy(synth.make_context(m, 35)).cuda()
    gm = GpuModel(m, synth.make_weights(m, init="stress"), proj=proj)
    v = gm.velocity(x, 0.5, ctx)
    for i in (0, 2047, 2048, n - 1):
        assert torch.equal(gm.velocity(x[i:i + 1], 0.5, ctx)[0], v[i]), i
    gm.close()
    del v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("name,n_cand", [("tiny", 16), ("wan_mid", 8)])
def test_rankings_are_those_of_the_compute_type(name, n_cand):
    """A score is a random projection of the latent, over the root of its size: scores differ by a normal value of the
    latents' difference in the mean square.  Five of its deviations are allowed, and swaps where the native gap is below
    twice that."""
    wl = synth.make_workload(name, init="paper", dtype=synth.DTYPE_BF16, n_cand=n_cand, mode=synth.CACHE_OFF)
    runs = []
    for proj in (B.CS_PROJ_8BIT, B.CS_PROJ_NATIVE):
        gm = GpuModel(wl.model, wl.weights, proj=proj)
        runs.append(run_rollout(gm, wl))
        gm.close()
    eight, native = runs
    off = np.sqrt(((eight.latents.astype(np.float64) - native.latents) ** 2).reshape(n_cand, -1).mean(-1))
    assert (np.abs(np.asarray(eight.scores) - native.scores) <= 5 * off).all()
    check_ranking(eight.scores, native.scores, 10 * off.max())
    print(name, "rho", B.cs_rank(eight.scores, native.scores)[2], "scores off", np.abs(np.asarray(eight.scores) - native.scores).max(),
          "latents", rel_l2(eight.latents, native.latents), flush=True)
