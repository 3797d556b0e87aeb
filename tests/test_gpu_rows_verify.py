"""Drafted tokens against the target's probabilities, sequence by sequence from the definition: whole numbers, equal."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2502_11517_amd import rows

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TOP = float(np.float32(1.0) - np.float32(2.0 ** -24))


def held(u):
    return min(max(float(u), 0.0), TOP) if u == u else 0.0


def one(p, q, token, draw, last, V):
    """(accepted, next token) of a sequence: p, q [n, V] float64"""
    n, a, rejected = len(token), 0, None
    for i in range(1, n):
        t = int(token[i])
        known = 0 <= t < V
        if known and held(draw[i]) * (q[i, t] if q is not None else 1.0) < p[i - 1, t]:
            a += 1
        else:
            rejected = t
            break
    finite = lambda x: np.where((x > 0) & (x < math.inf), x, 0.0)  # noqa: E731
    w = finite(p[a])
    if rejected is not None:
        with np.errstate(invalid="ignore"):
            rest = finite(p[a] - q[a + 1]) if q is not None else w.copy()
        if q is None and 0 <= rejected < V:
            rest[rejected] = 0.0
        if rest.sum() > 0:
            w = rest
    total = np.cumsum(w)
    if not total[-1] > 0:
        return a, -1
    return a, int(np.argmax((total > held(last) * total[-1]) & (w > 0)))


class Case:
    def __init__(self, seed, V, n_rows, dtype="f32", drafted=True, pad=0, apart=0.5, sharp=2.5, extra=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.V, self.rows, self.dtype = V, list(n_rows), dtype
        self.offs = np.concatenate([[0], np.cumsum(n_rows)]).astype(np.int32)
        self.S, self.n = len(self.rows), int(self.offs[-1]) + extra
        n = max(self.n, 1)
        x = sharp * torch.randn(n, V, device="cuda", generator=g)
        y = x.roll(1, 0) + apart * torch.randn(n, V, device="cuda", generator=g)
        wide = lambda z: torch.nn.functional.pad(torch.softmax(z, -1), (0, pad), value=0.7).to(TD[dtype])  # noqa: E731
        self.target, self.draft = wide(x), wide(y) if drafted else None
        self.token = torch.multinomial(torch.softmax(y, -1), 1, generator=g)[:, 0].int()
        self.draw, self.last = torch.rand(n, device="cuda", generator=g), torch.rand(max(self.S, 1), device="cuda", generator=g)
        self.length = torch.randint(50, 5000, (max(self.S, 1),), device="cuda", generator=g, dtype=torch.int32)
        self.position = torch.randint(0, 9000, (n,), device="cuda", generator=g, dtype=torch.int32)

    def out(self, k):
        return torch.full((max(k, 1),), -7, dtype=torch.int32, device="cuda")

    def run(self, stream=None, in_place=False, bare=False):
        cfg = rows.make_config(vocab=self.V, max_sequences=max(self.S, 1), max_rows=max(self.n, 1))
        ws = torch.full((rows.query_workspace_bytes(cfg),), 255, dtype=torch.uint8, device="cuda")
        offs = torch.from_numpy(self.offs).cuda()
        acc, nxt, keep = self.out(self.S), self.out(self.S), self.out(self.S)
        pos = self.position.clone()
        pos_out = pos if in_place else self.out(self.n)
        torch.cuda.synchronize()
        h = rows.PastaRows(cfg, ws, stream=(stream or torch.cuda.current_stream()).cuda_stream)
        more = {} if bare else dict(length=self.length, keep=keep, row_position=pos, position_out=pos_out)
        h.verify(offs, self.token, self.target, self.draw, self.last, acc, nxt, draft=self.draft, n_rows=self.n, **more)
        torch.cuda.synchronize()
        return [x.cpu().numpy() for x in (acc, nxt, keep, pos_out)]

    def want(self):
        p = self.target[:, :self.V].double().cpu().numpy()
        q = None if self.draft is None else self.draft[:, :self.V].double().cpu().numpy()
        token, draw, last, length = (x.cpu().numpy() for x in (self.token, self.draw, self.last, self.length))
        pos = self.position.cpu().numpy()
        acc, nxt, keep, pos_out = (np.full(max(k, 1), -7) for k in (self.S, self.S, self.S, self.n))
        end = min(max(int(self.offs[self.S]), 0), self.n)
        for s in range(self.S):
            lo = min(max(int(self.offs[s]), 0), end)
            hi = min(max(int(self.offs[s + 1]), lo), end)
            if lo == hi:
                acc[s], nxt[s], keep[s] = 0, -1, length[s]
                continue
            acc[s], nxt[s] = one(p[lo:hi], None if q is None else q[lo:hi], token[lo:hi], draw[lo:hi], last[s], self.V)
            keep[s] = length[s] - (hi - lo) + 1 + acc[s]
            pos_out[lo:hi] = pos[lo:hi] + 1 + acc[s]
        return acc, nxt, keep, pos_out

    def check(self, **kw):
        got, want = self.run(**kw), self.want()
        for name, g, w in zip(("accepted", "next_token", "keep", "position"), got, want):
            assert np.array_equal(g, w), (name, g, w)
        return got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 3, 5, 64, 255, 256, 257, 1000, 4095, 4097, 8192, 8193, 16385, 32000, 32768, 32769, 50001, 131072])
def test_vocabularies_of_every_size(V, dtype):
    got = Case(V, V, [5, 1, 3, 9, 2, 4], dtype).check()
    assert (got[0] >= 0).all() and (got[1] < V).all()


@pytest.mark.parametrize("V", [300, 40000])
@pytest.mark.parametrize("pad", [1, 3, 37])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_begin_anywhere(V, pad, dtype):
    Case(pad, V, [4, 2, 7], dtype, pad=pad).check()


@pytest.mark.parametrize("V", [300, 40000])
@pytest.mark.parametrize("apart", [0.0, 0.3, 5.0])
def test_drafts_that_were_chosen_and_drafts_that_were_drawn(V, apart):
    for drafted in (False, True):
        Case(11, V, [5] * 16, drafted=drafted, apart=apart, sharp=6.0).check()


@pytest.mark.parametrize("V", [300, 40000])
def test_sequences_without_rows_and_many_drafts(V):
    got = Case(12, V, [0, 1, 0, 70, 130, 0, 2], apart=0.0, sharp=3.0, extra=3).check()
    assert got[0][4] > 0


@pytest.mark.parametrize("V", [300, 40000])
def test_all_accepted_and_the_first_rejected(V):
    c = Case(13, V, [6, 6])
    c.draw[:6] = 0.0
    c.draw[6:] = 0.9999999
    c.target[6, c.token[7].long()] = 0.0
    got = c.check()
    assert got[0].tolist() == [5, 0] and got[2][0] == int(c.length[0]) and got[2][1] == int(c.length[1]) - 5


@pytest.mark.parametrize("V", [16, 4096, 65536])
def test_draws_on_a_border(V):
    """Uniform target, V a power of two: sums are exact, and a draw of t / V is the first of token t (the sum has to be above it)."""
    S = 64
    c = Case(14, V, [1] * S)
    c.target[:] = 1.0 / V
    t = torch.randint(0, V, (S,), device="cuda")
    t[:4] = torch.tensor([0, 1, V - 1, V // 2])
    c.last = t.float() / V
    got = c.check()
    assert np.array_equal(got[1], t.cpu().numpy())


@pytest.mark.parametrize("V", [300, 40000])
def test_acceptance_on_its_border(V):
    """draw * q < p: equal is rejected."""
    c = Case(15, V, [2, 2, 2])
    for s, u in enumerate((0.5, 0.5, 0.25)):
        t = int(c.token[2 * s + 1])
        c.draft[2 * s + 1, t], c.target[2 * s, t], c.draw[2 * s + 1] = 0.5, (0.25, 0.25 + 2.0 ** -25, 0.125)[s], u
    assert c.check()[0].tolist() == [0, 1, 0]


@pytest.mark.parametrize("V", [300, 40000])
@pytest.mark.parametrize("drafted", [True, False])
def test_tokens_outside_of_the_vocabulary_are_rejected(V, drafted):
    c = Case(16, V, [3, 3, 3, 3], drafted=drafted)
    c.token[torch.tensor([1, 4, 7, 10])] = torch.tensor([V, -1, 1 << 30, -(1 << 31)], dtype=torch.int32, device="cuda")
    c.token[torch.tensor([0, 3])] = torch.tensor([-5, 1 << 30], dtype=torch.int32, device="cuda")  # (a sequence's first row is not looked at)
    assert (c.check()[0] == 0).all()


@pytest.mark.parametrize("V", [300, 40000])
def test_where_the_target_is_nowhere_above_the_draft(V):
    """p = q but for the drafted token, which p does not know: nothing is left of p - q, and p itself is drawn from."""
    c = Case(17, V, [2, 2])
    for s in range(2):
        c.target[2 * s] = c.draft[2 * s + 1]
        c.target[2 * s, int(c.token[2 * s + 1])] = 0.0
    assert (c.check()[0] == 0).all()


@pytest.mark.parametrize("V", [300, 40000])
def test_weights_that_do_not_count(V):
    c = Case(18, V, [1, 1, 1, 3, 1])
    c.target[0] = 0.0
    c.target[1] = float("nan")
    c.target[2, ::3], c.target[2, 1::3] = float("inf"), -1.0
    c.target[3, ::2], c.draft[4, 1::5] = float("nan"), float("nan")
    c.target[6] = 0.0
    c.target[6, V - 1] = 1e-30
    got = c.check()
    assert got[1][0] == -1 and got[1][1] == -1 and got[1][2] % 3 == 2 and got[1][4] == V - 1


@pytest.mark.parametrize("V", [300, 20000, 40000])
def test_infinite_weights_beside_finite_ones(V):
    """Of p, of the draft's distribution (below p everywhere else, and nowhere), and where p alone is left."""
    c = Case(26, V, [2, 2, 2])
    t = c.token[[1, 3, 5]].long()
    c.target[[0, 2, 4], t] = 0.0  # (rejected)
    c.target[0, 7], c.draft[1, 11], c.draft[1, 12] = float("inf"), -float("inf"), float("inf")
    c.draft[3] = 2.0
    c.draft[3, 5] = -float("inf")
    c.draft[3, t[1]] = 1.0
    c.draft[5] = float("nan")
    c.draft[5, t[2]] = 1.0
    assert (c.check()[0] == 0).all()


@pytest.mark.parametrize("drafted", [True, False])
@pytest.mark.parametrize("V", [300, 20000, 40000])
def test_infinite_weights_where_the_draft_is_below_zero(V, drafted):
    """An infinite p less a negative q is infinite, too, and does not count, whatever the q."""
    c = Case(28, V, [2] * 8, drafted=drafted)
    t = c.token[1::2].long()
    c.target[:] = 0.0
    c.target[::2, 11] = 0.25
    c.target[::2, 7], c.target[::2, V - 1] = float("inf"), float("inf")
    c.token[1::2] = torch.where((t == 7) | (t == 11) | (t == V - 1), 8, t).int()  # (rejected: p is 0 there)
    if drafted:
        c.draft[:] = 0.0
        c.draft[1::2, 7], c.draft[1::2, V - 1] = -1000.0, -3.0e38
    got = c.check()
    assert (got[0] == 0).all() and (got[1] == 11).all()


@pytest.mark.parametrize("V", [300, 40000])
def test_draws_outside_of_their_range(V):
    c = Case(19, V, [1] * 6 + [2] * 3)
    c.last[:6] = torch.tensor([0.0, 1.0, -3.0, 7.0, float("nan"), float("inf")], device="cuda")
    c.draw[[7, 9, 11]] = torch.tensor([1.0, -1.0, float("nan")], device="cuda")
    c.check()


@pytest.mark.parametrize("V", [300, 40000])
def test_a_few_tokens_hold_everything(V):
    c = Case(20, V, [1] * 64)
    c.target[:] = 0.0
    g = torch.Generator(device="cuda").manual_seed(1)
    for k in range(3):
        c.target[torch.arange(64), torch.randint(0, V, (64,), device="cuda", generator=g)] = (0.25, 0.5, 2.0 ** -60)[k]
    c.last[:8] = torch.tensor([0.0, TOP, 0.5, 0.25, 2.0 / 3, 1.0 / 3, 1e-38, 0.999999], device="cuda")
    c.check()


@pytest.mark.parametrize("V", [300, 40000])
def test_sequences_that_were_refused_stay_as_they_are(V):
    c = Case(27, V, [4, 3, 1, 5])
    want = c.want()
    slot = torch.arange(c.n, dtype=torch.int32, device="cuda")
    slot[4:7], slot[7], slot[10] = -1, -1, -1  # (the last one: not a first row, which alone counts)
    cfg = rows.make_config(vocab=V, max_sequences=4, max_rows=c.n)
    ws = torch.empty(rows.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    acc, nxt, keep, pos = c.out(4), c.out(4), c.out(4), c.out(c.n)
    h = rows.PastaRows(cfg, ws, stream=torch.cuda.current_stream().cuda_stream)
    h.verify(torch.from_numpy(c.offs).cuda(), c.token, c.target, c.draw, c.last, acc, nxt, draft=c.draft, length=c.length, keep=keep, row_position=c.position,
             position_out=pos, slot=slot)
    torch.cuda.synchronize()
    length, position = c.length.cpu().numpy(), c.position.cpu().numpy()
    for s in (1, 2):
        want[0][s], want[1][s], want[2][s] = 0, -1, length[s]
        want[3][c.offs[s]:c.offs[s + 1]] = position[c.offs[s]:c.offs[s + 1]]
    for got, w in zip((acc, nxt, keep, pos), want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_offsets_that_are_wrong_stay_inside_the_arrays():
    for V in (300, 40000):
        c = Case(21, V, [3, 3, 3])
        for offs in ([0, 1 << 20, 3, 9], [-5, 4, 2, 9], [0, 3, 6, 1 << 30], [9, 9, 9, 9], [0, 0, 0, -1]):
            c.offs = np.array(offs, np.int32)
            acc, nxt, *_ = c.run()
            assert (acc >= 0).all() and (acc < 9).all() and (nxt >= -1).all() and (nxt < V).all()


def test_outputs_that_are_left_out_and_positions_in_place():
    c = Case(22, 5000, [3, 1, 4])
    want = c.want()
    got = c.run(bare=True)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]) and (got[2] == -7).all() and (got[3] == -7).all()
    assert np.array_equal(c.run(in_place=True)[3], want[3])


@pytest.mark.parametrize("V", [300, 40000])
def test_the_shares_of_the_tokens(V):
    """4096 draws in even steps over one distribution: token t gets its share of them, give or take one."""
    S = 4096
    c = Case(23, V, [1] * 8)
    p = c.target[0].double()
    p /= p.sum()
    cfg = rows.make_config(vocab=V, max_sequences=S, max_rows=S)
    ws = torch.empty(rows.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    h = rows.PastaRows(cfg, ws, stream=torch.cuda.current_stream().cuda_stream)
    many = c.target[:1].expand(S, V).contiguous()
    acc, nxt = c.out(S), c.out(S)
    h.verify(torch.arange(S + 1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda"), many, torch.zeros(S, device="cuda"),
             (torch.arange(S, device="cuda") + 0.5) / S, acc, nxt)
    count = torch.bincount(nxt.long(), minlength=V).double()
    assert (nxt.diff() >= 0).all() and ((count - p * S).abs() <= 1.0 + 1e-6).all()


def test_captured_and_replayed_on_another_stream():
    for V in (5000, 40000):
        c = Case(24, V, [4, 1, 6])
        s = torch.cuda.Stream()
        cfg = rows.make_config(vocab=V, max_sequences=3, max_rows=c.n)
        ws = torch.empty(rows.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        h = rows.PastaRows(cfg, ws, stream=s.cuda_stream)
        offs, acc, nxt = torch.from_numpy(c.offs).cuda(), c.out(3), c.out(3)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            h.verify(offs, c.token, c.target, c.draw, c.last, acc, nxt, draft=c.draft)
        for i in range(4):
            c.draw.copy_(torch.rand_like(c.draw))
            c.last.copy_(torch.rand_like(c.last))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want = c.want()
            assert np.array_equal(acc.cpu().numpy(), want[0]) and np.array_equal(nxt.cpu().numpy(), want[1])


def test_rows_behind_two_gibibytes():
    """Offsets of rows beyond 32 bits."""
    V, n = 131072, 4200
    c = Case(25, 131072, [2, 2])
    big = torch.zeros(n, V, device="cuda", dtype=torch.float32)
    big[-4:] = c.target[:4]
    draft = torch.zeros(n, V, device="cuda", dtype=torch.float32)
    draft[-4:] = c.draft[:4]
    cfg = rows.make_config(vocab=V, max_sequences=3, max_rows=n)
    h = rows.PastaRows(cfg, torch.empty(rows.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), stream=torch.cuda.current_stream().cuda_stream)
    token, draw = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    token[-4:], draw[-4:] = c.token[:4], c.draw[:4]
    last = torch.zeros(3, device="cuda")
    last[1:] = c.last[:2]
    acc, nxt = c.out(3), c.out(3)
    h.verify(torch.tensor([0, n - 4, n - 2, n], dtype=torch.int32, device="cuda"), token, big, draw, last, acc, nxt, draft=draft)
    torch.cuda.synchronize()
    want = c.want()
    assert np.array_equal(acc.cpu().numpy()[1:], want[0]) and np.array_equal(nxt.cpu().numpy()[1:], want[1]) and int(nxt[0]) == -1
