"""Codes of the stack of gated blocks and the answers that read them, on streams of their own: what is ordered behind what (no GPU: every stream carries the set of the calls that
are known to have ended before its next one, events and waits pass it on)."""
import contextlib
import threading

import pytest
import torch

from paper_1807_11205_amd import api, gated_mlp


class Event:
    seen = frozenset()


class Stream:
    def __init__(self, handle):
        self.cuda_stream, self.seen = handle, set()

    def wait_stream(self, other):
        self.seen |= other.seen

    def wait_event(self, event):
        self.seen |= event.seen

    def record_event(self, event=None):
        event = event or Event()
        event.seen = frozenset(self.seen)
        return event

    def synchronize(self):
        pass


class World:
    def __init__(self, monkeypatch):
        self.streams = {h: Stream(h) for h in (0, 7, 8, 9)}
        self.current, self.calls, self.capturing = self.streams[7], [], False

        @contextlib.contextmanager
        def on(s):
            before, self.current = self.current, s
            yield
            self.current = before
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: self.current)
        monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: self.streams[0])
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, *a: self.streams[h])
        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.capturing)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
        monkeypatch.setattr(gated_mlp.GatedMLP, "_buf", lambda m, shape, dtype=torch.float16: torch.zeros(shape, dtype=dtype))
        monkeypatch.setattr(api, "_stream", lambda s: (self.current if s is None else s).cuda_stream if s is None or hasattr(s, "cuda_stream") else int(s))
        for name in ("jz_quantize_i8", "jz_ffn_i8_fwd", "jz_linear_i8", "jz_norm_residual_fwd"):
            monkeypatch.setattr(api, name, lambda *a, name=name, stream=None, **k: self.call(name, stream))

    def call(self, name, stream):
        s = self.current if stream is None else self.streams[api._stream(stream)]
        n = len(self.calls)
        self.calls.append((name, frozenset(s.seen)))
        s.seen.add(n)

    def since(self, first, *names):
        return {n for n in range(first, len(self.calls)) if self.calls[n][0] in names}


READS = ("jz_ffn_i8_fwd", "jz_linear_i8")


def stack():
    m = gated_mlp.GatedMLP.__new__(gated_mlp.GatedMLP)
    m.width, m.hidden, m.classes, m.blocks, m.scale, m.device = 16, 32, 8, 2, 0.5, torch.device("cpu")
    m.shapes = {"%s_%d" % (n, i): (16, 32) if n == "w_down" else (32, 16) for n in ("w_gate", "w_up", "w_down") for i in range(2)}
    m.shapes["w_fc"] = (8, 16)
    m.master = m.w16 = torch.zeros(1)
    m.i8_lock = threading.Lock()
    m._param = lambda buf, name: buf
    return m


@pytest.mark.parametrize("codes", [None, 8, "eight"])
@pytest.mark.parametrize("answers", [None, 9, "nine"])
def test_answers_wait_for_the_codes_and_new_codes_for_the_answers(monkeypatch, codes, answers):
    w, m = World(monkeypatch), stack()
    pick = lambda s: w.streams[{"eight": 8, "nine": 9}[s]] if isinstance(s, str) else s
    written = set()
    for _ in range(3):
        first = len(w.calls)
        m.prepare_answers_i8(stream=pick(codes))
        new = w.since(first, "jz_quantize_i8")
        read = w.since(0, *READS)
        assert len(new) == 7 and all(read | written <= w.calls[n][1] for n in new)
        written |= new
        first = len(w.calls)
        for s in (pick(answers), None, 8):
            m.answer(torch.zeros(3, 16), s, i8=True)
        reads = w.since(first, *READS)
        assert len(reads) == 9 and all(written <= w.calls[n][1] for n in reads)


def test_codes_written_from_two_streams(monkeypatch):
    w, m = World(monkeypatch), stack()
    m.prepare_answers_i8(stream=8)
    m.prepare_answers_i8(stream=9)
    assert all(set(range(7)) <= w.calls[n][1] for n in range(7, 14))


def test_a_capture_waits_for_nothing_outside(monkeypatch):
    w, m = World(monkeypatch), stack()
    m.prepare_answers_i8(stream=8)
    w.capturing = True
    first = len(w.calls)
    m.answer(torch.zeros(3, 16), i8=True)
    m.prepare_answers_i8()
    assert all(not (set(range(first)) & seen) for _, seen in w.calls[first:])
    w.capturing = False
    m.answer(torch.zeros(3, 16), i8=True)       # waits for the codes of before the capture, as if that had not been
    assert set(range(7)) <= w.calls[-1][1]


def test_codes_from_a_thread_wait_for_the_answer_that_is_being_launched(monkeypatch):
    """One thread answers while another writes new codes: all launches of either lie together, and the later ones behind the earlier ones' event."""
    w, m = World(monkeypatch), stack()
    m.prepare_answers_i8()
    first, thread = len(w.calls), []

    def between(*a, stream=None, **k):      # in the middle of the answer
        if not thread:
            thread.append(threading.Thread(target=m.prepare_answers_i8, kwargs=dict(stream=8)))
            thread[0].start()
            thread[0].join(0.3)
        w.call("jz_ffn_i8_fwd", stream)
    monkeypatch.setattr(api, "jz_ffn_i8_fwd", between)
    m.answer(torch.zeros(3, 16), 9, i8=True)
    thread[0].join()
    reads, new = w.since(first, *READS), w.since(first, "jz_quantize_i8")
    assert len(reads) == 3 and len(new) == 7 and all(reads <= w.calls[n][1] for n in new)
