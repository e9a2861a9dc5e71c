"""On which stream stack.ExpertShard and TokenTrainStep work when one is given as a torch
stream, as its number or as the default stream's number, 0: with torch's streams
replaced by a record, and on the GPU against the step on the current stream."""
import contextlib

import numpy as np
import pytest
import torch

from paper_2112_15317_amd import stack
from tests.helpers import print_case


class Stream:
    def __init__(self, number):
        self.cuda_stream = number


@pytest.mark.parametrize("kind,want", [("none", None), ("stream", 7), ("number", 7), ("default", 0)])
def test_the_stream_that_is_made_current(monkeypatch, kind, want):
    entered = []

    @contextlib.contextmanager
    def on(stream):
        entered.append(stream.cuda_stream)
        yield
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: Stream(0))
    # Of 0 torch makes a stream of its own pool.
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda n: Stream(n or 99))
    with stack._on({"none": None, "stream": Stream(7), "number": 7, "default": 0}[kind]):
        pass
    assert entered == ([] if want is None else [want])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["stream", "number", "default"])
def test_a_step_on_a_given_stream(kind):
    print_case("token step on a stream", kind=kind)
    tokens, vocab = 200, 900
    r = np.random.default_rng(1)
    ids, targets = (torch.from_numpy(r.integers(0, vocab, tokens).astype(np.int32)) for _ in range(2))
    got = []
    for given in (None, kind):
        step = stack.TokenTrainStep(tokens, vocab, 48, 40, 5, 2, stack.AdamW(lr=1e-3), alternatives=3)
        q = np.random.default_rng(2)
        for w, _, _, _ in step.params.items:
            step.params.load(w, q.normal(size=tuple(w.shape)) * 0.3)
        step.ids.copy_(ids)
        step.targets.copy_(targets)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        step.step({None: None, "stream": side, "number": side.cuda_stream,
                   "default": torch.cuda.default_stream().cuda_stream}[given])
        torch.cuda.synchronize()
        got.append([step.logp, step.entropy, step.top_ids] + [t for w, g, _, _ in step.params.items for t in (w, g)])
    assert all(torch.equal(a, b) for a, b in zip(*got))
