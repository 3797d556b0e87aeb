"""Drafts that a session takes back, without a GPU: slots by the walk request by request (kv8_ref), verify by its definition, on host tensors."""
from __future__ import annotations

import contextlib

import numpy as np
import pytest
import torch

import kv8_ref as ref
from paper_2502_11517_amd import kv8_session
from paper_2502_11517_amd.kv8_session import Session, _Request

P, W, R = 16, 30, 2


class Slots:
    """The handle: places as the library gives them."""

    def __init__(self, s, pages):
        self.s, self.table, self.stack = s, np.full((R, W), -1), np.arange(pages - 1, -1, -1)
        s.free_count = torch.tensor([pages], dtype=torch.int32)

    def slots(self, length, offsets, n, slot, length_out, free_count, free_out, *, keep=None, row_tag=None, row_position=None):
        got = ref.slots(P, W, length.numpy(), None if keep is None else keep.numpy(), offsets.numpy(), n, self.table, self.stack, int(free_count))
        if n:
            slot[:n] = torch.from_numpy(got[0]).int()
        length_out.copy_(torch.from_numpy(got[1]).int())
        free_out.fill_(int(got[2]))
        self.table, self.stack = got[3], got[4]

    def plan(self, *args, **kw):
        pass


class Verify:
    """The rows' handle: as many drafts of each request accepted as `self.accept` says."""

    accept = (0, 0)

    def verify(self, offsets, token, target, draw, last_draw, accepted, next_token, *, length, keep, row_position, position_out, slot, n_rows, **kw):
        for r in range(R):
            lo, hi = int(offsets[r]), int(offsets[r + 1])
            refused = hi > lo and int(slot[lo]) < 0
            a = 0 if refused or hi == lo else min(self.accept[r], hi - lo - 1)
            accepted[r], next_token[r] = a, -1 if refused or hi == lo else 1
            keep[r] = int(length[r]) if refused or hi == lo else int(length[r]) - (hi - lo) + 1 + a
            position_out[lo:hi] = row_position[lo:hi] + (0 if refused else 1 + a)


@pytest.fixture
def session(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())

    def made(pages):
        s = object.__new__(Session)
        s.device, s._stream, s._step, s._captured, s.slopes, s.logit_cap = torch.device("cpu"), None, None, [], None, 0.0
        s.requests = [_Request() for _ in range(R)]
        i32 = dict(dtype=torch.int32)
        s.length, s.prefix_len, s.keep, s.accepted = (torch.zeros(R, **i32) for _ in range(4))
        s._no_rows = torch.zeros(R + 1, **i32)
        s.next_token, s.slot = torch.full((R,), -1, **i32), torch.full((64,), -1, **i32)
        s.handle, s.rows = Slots(s, pages), Verify()
        s.threads = [s.open(r) for r in range(R)]
        return s
    return made


def verify(s, *accept):
    s.rows.accept = accept
    s.verify(None, None, None, None)


def state(s):
    return s.length.tolist(), s.keep.tolist(), [t.position for t in s.threads]


@pytest.mark.parametrize("waits", ["again", "begin", "begin of another", "twice"])
def test_a_refused_step_behind_a_verified_one_keeps_no_rejected_drafts(session, waits):
    """27 tokens and five rows of which two drafts are accepted: 30 tokens of 32.  Five more rows want a third page, which the other request holds."""
    s, free = session(3), session(60)
    for x in (s, free):
        one, other = x.threads
        x.begin([one] * 27 + [other] * 16)
        x.begin([one] * 5)
        verify(x, 2, 0)
        assert x.settle() == [2, 0] and one.position == 30
    one = s.threads[0]
    if waits == "begin of another":  # (which is served, and takes the drafts back as well)
        s.threads[1].position = 0
        s.release(1)
        s.threads[1] = s.open(1)
        s.begin([s.threads[1]] * 16)
        assert s.length.tolist() == [30, 16]
    for _ in range(2 if waits == "twice" else 1):
        if waits == "again":
            s.again()
        else:
            s.begin([one] * 5)
        assert s.slot[:5].tolist() == [-1] * 5
        verify(s, 4, 0)
        assert s.refused() == [0] and s.settle()[0] == 0 and one.position == 30
    s.release(1)
    assert s.length.tolist() == [30, 0]
    for x in (s, free):
        if x is free:
            x.release(1)
        x.begin([x.threads[0]] * 5)
        verify(x, 1, 0)
        x.settle()
        x.begin([x.threads[0]] * 3)
    assert state(s)[0] == state(free)[0] == [30 + 2 + 3, 0] and state(s)[2][0] == state(free)[2][0] == 35


def test_a_refused_step_that_is_not_verified(session):
    s = session(3)
    one, other = s.threads
    s.begin([one] * 27 + [other] * 16)
    s.begin([one] * 5)
    verify(s, 2, 0)
    s.again()  # refused
    assert s.refused() == [0]
    s.settle()
    s.release(1)
    s.begin([one])
    assert s.length.tolist() == [31, 0] and s._step["position"].tolist() == [30]


def test_a_page_of_rejected_drafts_goes_back_ahead_of_the_step(session):
    """The second request's five rows take the last page, and none is accepted: in the next step the first request gets it, which comes first."""
    s = session(3)
    one, other = s.threads
    s.begin([one] * 16 + [other] * 15)
    s.settle()
    s.begin([other] * 5)
    verify(s, 0, 0)
    s.settle()
    assert s.length.tolist() == [16, 20] and int(s.free_count) == 0 and other.position == 16
    s.begin([one, other])
    assert s.length.tolist() == [17, 16] and s.refused() == [1] and other.position == 16


def test_settle_goes_by_captured_steps_whose_threads_went_on_nowhere_else(session, monkeypatch):
    s = session(60)
    one, other = s.threads
    for t in (one, other):
        s.begin([t] * 4)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
        s.again()
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
        verify(s, 1, 1)
        s.settle()
    assert [c["verified"] for c in s._captured] == [True, True] and (one.position, other.position) == (6, 6)
    s.begin([one])
    assert [c["verified"] for c in s._captured] == [False, True]
    s.settle()
    assert (one.position, other.position) == (7, 6)
    s.again()
    assert [c["verified"] for c in s._captured] == [False, True]
