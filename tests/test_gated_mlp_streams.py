"""Which stream everything in the answers of the stack of gated blocks belongs to (no GPU: streams, allocations and the library's calls are recorded)."""
import contextlib
import inspect

import pytest
import torch

from paper_1807_11205_amd import api, gated_mlp


class Stream:
    def __init__(self, handle):
        self.cuda_stream, self.waits = handle, []

    def wait_stream(self, other):
        self.waits.append(other)


class World:
    """What happens, and on which stream: (what, stream's handle)."""

    def __init__(self, monkeypatch):
        self.current, self.log, self.used = Stream(7), [], []
        self.home = self.current

        @contextlib.contextmanager
        def on(s):
            before, self.current = self.current, s
            yield
            self.current = before
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.current)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: Stream(0))
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, *a: Stream(h))
        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: self.used.append((t, s.cuda_stream)))
        for name in ("clone", "to"):
            real = getattr(torch.Tensor, name)
            monkeypatch.setattr(torch.Tensor, name, lambda t, *a, real=real, name=name, **k: self.at(name) or real(t, *a, **k))
        monkeypatch.setattr(gated_mlp.GatedMLP, "_buf", lambda m, shape, dtype=torch.float16: self.at("buffer") or torch.zeros(shape, dtype=dtype))
        monkeypatch.setattr(api, "_stream", lambda s: (self.current if s is None else s).cuda_stream if s is None or hasattr(s, "cuda_stream") else int(s))
        for name in ("jz_norm_residual_fwd", "jz_ffn_fwd", "jz_gemm_fc"):
            binds = inspect.signature(getattr(api, name)).bind
            monkeypatch.setattr(api, name, lambda *a, binds=binds, name=name, **k: self.log.append((name, api._stream(binds(*a, **k).arguments.get("stream")))))

    def at(self, what):
        self.log.append((what, self.current.cuda_stream))


def stack():
    m = gated_mlp.GatedMLP.__new__(gated_mlp.GatedMLP)
    m.width, m.hidden, m.classes, m.blocks, m.scale, m.device = 16, 32, 8, 2, 0.5, torch.device("cpu")
    m.master = m.w16 = torch.zeros(1)
    m._param = lambda buf, name: buf
    return m


@pytest.mark.parametrize("stream", [None, Stream(7), Stream(9), 9, 0])
def test_answers_belong_to_one_stream(monkeypatch, stream):
    w, m = World(monkeypatch), stack()
    x = torch.zeros(3, 16)
    out = m.answer(x, stream) if stream is not None else m.answer(x)
    want = 7 if stream is None else getattr(stream, "cuda_stream", stream)
    assert [s for s in w.log if s[1] != want] == []
    assert {k for k, _ in w.log} == {"clone", "to", "buffer", "jz_norm_residual_fwd", "jz_ffn_fwd", "jz_gemm_fc"}
    assert w.current is w.home
    if want != 7:           # x is read on the other stream, the logits are read on this one
        assert any(t is x and s == want for t, s in w.used) and any(t is out and s == 7 for t, s in w.used)
    if isinstance(stream, Stream) and want != 7:
        assert stream.waits == [w.home]
