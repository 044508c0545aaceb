"""Who frees a model's prompts, and in which order (no GPU needed: the library is stood in for)."""
import gc
import weakref

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_23159_amd import search, synth


@pytest.fixture
def freed(monkeypatch):
    """Order in which handles are freed; models are 1, 2, ..., contexts 101, 102, ..."""
    log, n = [], {"m": 0, "c": 100}

    def make(kind):
        def f(*args):
            n[kind] += 1
            return n[kind]
        return f
    monkeypatch.setattr(search, "_dev", lambda a: a)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    monkeypatch.setattr(search.B, "cs_model_init_norm", make("m"))
    monkeypatch.setattr(search.B, "cs_context_init", make("c"))
    monkeypatch.setattr(search.B, "cs_model_free", lambda h: log.append(h))
    monkeypatch.setattr(search.B, "cs_context_free", lambda h: log.append(h))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream(0, []))
    yield log
    for gm in _models:                 # a failed test's frames keep theirs: nothing real may be freed
        gm.contexts, gm.h = set(), 0
    _models.clear()


_models = weakref.WeakSet()


class Stream:
    def __init__(self, handle, log):
        self.cuda_stream, self.log = handle, log

    def synchronize(self):
        self.log.append("wait")


def _model(stream=None):
    m = synth.MODELS["tiny"]
    gm = search.GpuModel(m, np.zeros(synth.weight_count(m), np.float32), stream=stream)
    _models.add(gm)
    return gm


def test_a_model_closed_first_frees_its_prompts_before_itself(freed):
    gm = _model()
    a, b, c = (gm.prompts(torch.zeros(1)) for _ in range(3))
    b.close()
    gm.close()
    assert freed[0] == 102 and sorted(freed[1:3]) == [101, 103] and freed[3:] == [1]
    for p in (a, b, c):
        p.close()                      # nothing twice
    gm.close()
    assert len(freed) == 4


def test_prompts_closed_or_dropped_first(freed):
    gm = _model()
    with_close, dropped = gm.prompts(torch.zeros(1)), gm.prompts(torch.zeros(1))
    with_close.close()
    del dropped
    gc.collect()
    assert freed == [101, 102]
    gm.close()
    assert freed == [101, 102, 1]


def test_a_model_and_prompts_that_go_together(freed):
    """In a cycle of references, whichever is finalised first."""
    gm = _model()
    gm.mine = gm.prompts(torch.zeros(1))
    del gm
    gc.collect()
    assert freed == [101, 1]


@pytest.mark.parametrize("model_stream,current,waits", [(None, 0, False), (None, 8, True), (8, 8, False), (8, 0, True),
                                                        (Stream(8, []), 8, False), (Stream(8, []), 16, True)])
def test_prompts_wait_for_inputs_of_another_stream(freed, monkeypatch, model_stream, current, waits):
    """The library works on the model's stream: what the current one still has to produce is waited for."""
    log = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream(current, log))
    monkeypatch.setattr(search.B, "cs_context_init", lambda *args: log.append("init") or 101)
    monkeypatch.setattr(search.B, "cs_velocity_context", lambda *args: log.append("velocity"))
    gm = _model(model_stream)
    ps = gm.prompts(torch.zeros(1))
    ps.velocity(torch.zeros(1, 4), 0.5)
    assert log == (["wait", "init", "wait", "velocity"] if waits else ["init", "velocity"])
