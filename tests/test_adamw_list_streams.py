"""On which stream sb.AdamwList takes the memory of its plan, writes it and waits for
it, with torch's streams replaced by a record: nothing is launched."""
import contextlib

import pytest
import torch

from paper_2112_15317_amd import sb


class Stream:
    def __init__(self, number, capturing=False):
        self.cuda_stream, self.capturing, self.waits = number, capturing, 0

    def synchronize(self):
        self.waits += 1


class Record:
    """The current stream, and what was done on which."""

    def __init__(self, monkeypatch, capturing=False):
        self.current = self.first = Stream(0, capturing)
        self.at, self.written = [], []
        made = torch.empty

        def empty(*args, **kw):
            self.at.append(self.current.cuda_stream)
            return made(*args, **kw)

        @contextlib.contextmanager
        def on(stream):
            before, self.current = self.current, stream
            yield
            self.current = before

        lib = sb.load()

        class Lib:
            sb_adamw_plan_bytes = lib.sb_adamw_plan_bytes

            @staticmethod
            def sb_adamw_make_plan(*args):
                self.written.append(args[-1])
                return sb.SB_OK
        set_ = monkeypatch.setattr
        set_(torch, "empty", empty)
        set_(torch.cuda, "Stream", Stream)
        set_(torch.cuda, "ExternalStream", Stream)
        set_(torch.cuda, "stream", on)
        set_(torch.cuda, "current_stream", lambda *a: self.current)
        set_(torch.cuda, "synchronize", lambda *a: None)
        set_(torch.cuda, "is_current_stream_capturing", lambda: self.current.capturing)
        set_(sb, "load", lambda: Lib)
        set_(sb, "_ptr", lambda t: t if t is None or isinstance(t, int) else t.data_ptr())
        set_(sb, "_stream_for", lambda t, stream: (stream or self.current).cuda_stream)


def _items():
    z = [torch.zeros(8) for _ in range(4)]
    return [dict(zip("wgmv", z))]


@pytest.mark.parametrize("kind", ["none", "stream", "number"])
def test_memory_writing_and_wait_are_one_streams(monkeypatch, kind):
    rec = Record(monkeypatch)
    s = Stream(7)
    made = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda n: made.append(Stream(n)) or made[-1])
    sb.AdamwList(_items(), stream={"none": None, "stream": s, "number": 7}[kind])
    want = rec.first if kind == "none" else made[0] if kind == "number" else s
    assert rec.at == rec.written == [want.cuda_stream]
    assert want.waits == 1 and rec.current is rec.first


def test_the_captured_stream_is_not_waited_for(monkeypatch):
    rec = Record(monkeypatch, capturing=True)
    sb.AdamwList(_items())
    s = Stream(7, capturing=True)                    # joined to the capture
    sb.AdamwList(_items(), stream=s)
    assert rec.at == rec.written == [0, 7] and rec.first.waits == s.waits == 0


def test_a_stream_outside_the_capture_is_refused(monkeypatch):
    rec = Record(monkeypatch, capturing=True)
    s = Stream(7)
    with pytest.raises(ValueError, match="capture"):
        sb.AdamwList(_items(), stream=s)
    assert rec.written == [] and s.waits == 0
    # A stream that is captured while the current one is not.
    rec = Record(monkeypatch)
    s = Stream(7, capturing=True)
    sb.AdamwList(_items(), stream=s)
    assert rec.written == [7] and s.waits == rec.first.waits == 0
