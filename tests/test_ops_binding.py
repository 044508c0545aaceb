"""What the binding of the stand-alone operators hands to the library (no GPU needed: the
library and torch's device calls are stood in for)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2607_23159_amd import binding as B

CURRENT, P = 0x5150, 1 << 20
DEV = torch.device("cuda", 0)


class Recorder:
    """A library whose calls succeed and leave their arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return B.CS_OK
        return call


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(B, "lib", lambda: r)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: CURRENT + index, raising=False)
    return r


def _desc(struct, *names):
    return B._OpDesc(struct, **{n: (torch.bfloat16, torch.Size([1]), (1,), DEV) for n in names})


class FakeRows:
    """Rows, their cache's descriptor among them, that only have an address."""
    def data_ptr(self):
        return P


class FakeCache:
    device = DEV
    c = B.cs_kv4_cache()
    ref = C.byref(c)

    def rows(self, k, v):
        return _desc(B.cs_kv4_rows(n_rows=1), "k")


def _calls(stream):
    norm = _desc(B.cs_qk_norm_desc(tokens=1), "q", "k", "q_out", "k_out", "q_gain", "k_gain", "rope")
    attn = _desc(B.cs_attn_desc(n_q=1, n_kv=1, lk=1), "q", "k", "v", "o")
    kw = {} if stream is None else dict(stream=stream)
    B.cs_qk_norm_rope(norm, P, P, P, P, P, P, P, **kw)
    B.cs_kv4_store(FakeCache(), FakeRows(), FakeRows(), **kw)
    B.cs_kv4_load(FakeCache(), FakeRows(), FakeRows(), **kw)
    B.cs_cross_attention(attn, P, P, P, P, **kw)
    B.cs_kv4_attention(attn, P, FakeCache(), P, **kw)


def test_operators_run_on_the_current_stream_or_the_given_one(recorder):
    class Stream:
        cuda_stream = 77
    for stream, want in ((None, CURRENT), (Stream(), 77), (0, 0), (4096, 4096)):
        recorder.calls.clear()
        _calls(stream)
        assert [n for n, _ in recorder.calls] == ["cs_qk_norm_rope", "cs_kv4_store", "cs_kv4_load", "cs_cross_attention",
                                                  "cs_kv4_attention"]
        assert [args[-1] for _, args in recorder.calls] == [want] * 5


class FakeMask:
    is_cuda, device, dtype = True, DEV, torch.uint8

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P


def test_a_mask_whose_rows_are_longer_than_the_contexts_is_refused(recorder):
    """Its rows would be read lk apart, across its own."""
    attn = _desc(B.cs_attn_desc(n_q=2, n_kv=2, lk=40), "q", "k", "v", "o")
    for call in (lambda m: B.cs_cross_attention(attn, P, P, P, P, kv_mask=m),
                 lambda m: B.cs_kv4_attention(attn, P, FakeCache(), P, kv_mask=m)):
        for shape in ((2, 48), (40, 2), (2, 1, 80), (1, 2, 41), (1, 40), (79,)):
            with pytest.raises(ValueError, match="kv_mask"):
                call(FakeMask(*shape))
        recorder.calls.clear()
        for shape in ((2, 40), (3, 40), (2, 1, 40), (80,)):
            call(FakeMask(*shape))
        assert len(recorder.calls) == 4
