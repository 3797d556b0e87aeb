"""What a session keeps on the host, without a GPU: its calls go to a stand-in that writes them down."""
from __future__ import annotations

import gc
import weakref

import pytest
import torch

from paper_2502_11517_amd import kv8_session
from paper_2502_11517_amd.kv8_session import Session, _Request


class Calls:
    """The handle's calls, accepted unless told otherwise."""

    def __init__(self):
        self.made, self.refuse = [], None

    def __getattr__(self, name):
        if name.startswith("__"):
            raise AttributeError(name)

        def call(*args, **kw):
            if self.refuse == name:
                raise kv8_session.kv8.PastaError(kv8_session.kv8.E_CAPACITY, name)
            self.made.append((name, args, kw))
        return call


@pytest.fixture
def session(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    s = object.__new__(Session)
    s.device, s._stream, s._step, s._captured, s.slopes, s.logit_cap = torch.device("cpu"), None, None, [], None, 0.0
    s.handle, s.requests = Calls(), [_Request() for _ in range(3)]
    s.length, s.prefix_len, s.free_count = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    s.slot = torch.full((16,), -1, dtype=torch.int32)
    return s


def test_a_captured_steps_memory_outlives_the_steps_that_follow(session, monkeypatch):
    t = session.open(0)
    session.begin([t] * 3)
    gone = weakref.ref(session._step["offsets"])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    session.again()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    kept = [weakref.ref(v) for v in session._step.values() if torch.is_tensor(v)]
    assert len(kept) == 5
    u = session.open(1)
    session.begin([u])
    between = weakref.ref(session._step["offsets"])
    session.begin([u])
    gc.collect()
    assert gone() is not None and all(r() is not None for r in kept)
    session.handle.made.clear()
    gc.collect()
    assert between() is None and all(r() is not None for r in kept)
