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


def test_a_bound_steps_old_memory_waits_for_the_copies(session, monkeypatch):
    """The copies are made on the new stream, and the allocator knows memory by the stream it was taken on."""
    import contextlib

    waits = []

    class Recorded(torch.Tensor):
        def record_stream(self, stream):
            waits.append((self.data_ptr(), stream))

    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(kv8_session.kv8, "PastaKv8", lambda *args, **kw: Calls())
    for name in ("cfg", "workspace", "page_table", "k_codes", "v_codes", "k_scale", "v_scale", "free_pages", "slot_tag", "slot_position"):
        setattr(session, name, None)
    t = session.open(0)
    session.begin([t] * 4)
    session._step = {k: v.as_subclass(Recorded) if torch.is_tensor(v) else v for k, v in session._step.items()}
    old = [v.data_ptr() for v in session._step.values() if torch.is_tensor(v)]

    class Stream:
        cuda_stream = 7

    new = Stream()
    session.bind(new)
    assert sorted(waits, key=lambda w: w[0]) == [(p, new) for p in sorted(old)] and len(old) == 5
    assert not set(old) & {v.data_ptr() for v in session._step.values() if torch.is_tensor(v)}


@pytest.mark.parametrize("refuse", ["slots", "plan", "positions"])
def test_a_step_that_is_not_accepted_moves_nothing_on(session, refuse):
    t = session.open(0)
    session.begin([t] * 5)
    u = session.fork(t)
    before = session._step
    session.handle.refuse = refuse
    with pytest.raises((kv8_session.kv8.PastaError, IndexError)):
        session.begin([t, u, t, u], positions=[9, 9] if refuse == "positions" else None)
    assert (t.position, u.position) == (5, 5) and session._step is before
    session.handle.refuse = None
    session.begin([t, u, t, u])
    assert (t.position, u.position) == (7, 7) and session._step["position"].tolist() == [5, 5, 6, 6] and session._step["stride"].tolist() == [2] * 4
    session.begin([u, t, u], positions=[40, 3, 50])
    assert (t.position, u.position) == (4, 51)


def test_positions_of_refused_requests_are_set_back(session):
    a, b = session.open(0), session.open(1)
    session.begin([a] * 2 + [b] * 3)
    session.slot[:5] = torch.tensor([0, 1, 16, 17, 18])
    assert session.refused() == [] and (a.position, b.position) == (2, 3)
    kid = session.fork(b)
    session.begin([a, b, kid, b, kid])
    assert session._step["position"].tolist() == [2, 3, 3, 4, 4]
    session.slot[:5] = torch.tensor([2, -1, -1, -1, -1])
    assert (a.position, b.position, kid.position) == (3, 5, 5)
    for _ in range(2):
        assert session.refused() == [1] and (a.position, b.position, kid.position) == (3, 3, 3)
    session.again()
    session.advanced([a, b, kid, b, kid], 1)
    assert session._step["position"].tolist() == [3, 3, 3, 4, 4] and (a.position, b.position, kid.position) == (4, 5, 5)
    session.slot[:5] = torch.tensor([-1, 19, 20, 21, 22])
    assert session.refused() == [0] and (a.position, b.position, kid.position) == (3, 5, 5)


def test_a_layers_launches_are_made_under_the_sessions_device(session, monkeypatch):
    import contextlib

    under = []

    @contextlib.contextmanager
    def device(d):
        under.append(d)
        yield
        under.append(len(session.handle.made))

    session.begin([session.open(0)])
    session.handle.made.clear()
    monkeypatch.setattr(torch.cuda, "device", device)
    session.layer(0, None, None, None, None)
    assert under == [session.device, 2] and [name for name, _, _ in session.handle.made] == ["append", "attend"]


def test_threads_that_have_ended_neither_join_nor_fork(session):
    root = session.open(0)
    a, b, c = (session.fork(root) for _ in range(3))
    session.join(root, [a])
    before = [(t.tag, t.sees, t.alive) for t in (root, a, b, c)], session.requests[0].used
    for call in (lambda: session.join(a, [b, c]), lambda: session.join(a, [b, root, c]), lambda: session.join(root, [b, b]), lambda: session.join(root, [b, a]),
                 lambda: session.join(b, [c, b]), lambda: session.fork(a)):
        with pytest.raises(ValueError):
            call()
        assert before == ([(t.tag, t.sees, t.alive) for t in (root, a, b, c)], session.requests[0].used) and session.requests[0].threads == [root, b, c]
    session.join(root, (t for t in (b, c)))  # anything that can be gone over once
    assert not b.alive and not c.alive and session.requests[0].threads == [root] and session.requests[0].used == 1
    session.release(0)
    with pytest.raises(ValueError):
        session.fork(root)
