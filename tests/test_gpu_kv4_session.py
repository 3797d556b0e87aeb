"""The operators together: threads that fork and join over the 4-bit cache; q and k turned on their way; drafts verified and taken back, called step by
step and replayed from a graph, over both caches."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2502_11517_amd import kv4, rows
from paper_2502_11517_amd.kv8_session import Session
from test_gpu_kv8_session import Watched

pytestmark = pytest.mark.gpu


class Watched4(Watched):
    def __init__(self, seed, **kw):
        super().__init__(seed, codes="e2m1", **kw)

    def values(self):
        s = self.s
        return ref.Cache.unpack(s.cfg.n_phys_pages, s.cfg.n_kv_heads, s.cfg.page_tokens, s.cfg.head_dim,
                                *(b[0].cpu().numpy() for b in (s.k_codes, s.v_codes, s.k_scale, s.v_scale))).natural()


@pytest.mark.parametrize("dtype,D,seed", [("bf16", 64, 1), ("f16", 64, 2), ("bf16", 128, 3)])
def test_random_forks_and_joins(dtype, D, seed):
    w = Watched4(seed, dtype=dtype, head_dim=D)
    rng = w.rng
    live = [[w.open(r)] for r in range(3)]
    w.step([t for r in range(3) for t in live[r] * int(rng.integers(1, 60))])
    for _ in range(25):
        what = rng.random()
        r = int(rng.integers(0, 3))
        if what < 0.3 and len(live[r]) < 6:
            live[r].append(w.fork(live[r][int(rng.integers(0, len(live[r])))]))
        elif what < 0.45 and len(live[r]) > 1:
            n = int(rng.integers(1, len(live[r])))
            w.join(live[r][0], live[r][1:1 + n])
            del live[r][1:1 + n]
        step = [t for r in range(3) for t in live[r] if rng.random() < 0.8]
        if step:
            w.step(step)


def test_a_released_requests_pages_come_back():
    w = Watched4(5)
    a, b = w.open(0), w.open(1)
    w.step([a] * 100 + [b] * 20)
    left = int(w.s.free_count)
    w.s.release(0)
    w.rows[0] = 0
    w.step([b])
    assert int(w.s.free_count) == left + 7 and w.s.length.cpu().tolist()[:2] == [0, 21]
    w.step([w.open(0)] * 30)


SIZES = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, softmax_scale=0.125, n_layers=2, max_requests=2, max_rows=256, n_phys_pages=60, pages_per_request=30)


@pytest.mark.parametrize("codes", ["e2m1", "e4m3"])
def test_rope_turns_what_a_program_would_turn_itself(codes):
    f, m = rows.rope_frequencies(32, scaling="parts", factor=8.0)
    rope = dict(rope_dims=32, rope_layout="interleaved", rope_frequency=f, rope_magnitude=m)
    a, b = Session(codes=codes, rope=rope, **SIZES), Session(codes=codes, **SIZES)
    h = rows.PastaRows(rows.make_config(max_rows=256, n_q_heads=8, n_kv_heads=2, head_dim=64, **rope), stream=torch.cuda.current_stream().cuda_stream)
    g = torch.Generator(device="cuda").manual_seed(1)
    ta, tb = a.open(0), b.open(0)
    for n, ids in ((20, None), (3, [500, 501, 90]), (1, None)):
        x = lambda k: torch.randn(n, k, 64, device="cuda", generator=g).bfloat16()  # noqa: E731
        a.begin([ta] * n, ids)
        b.begin([tb] * n, ids)
        for l in range(2):
            q, k, v = x(8), x(2), x(2)
            oa, ob, qt, kt = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
            a.layer(l, k, v, q, oa)
            h.rotate(b._step["position"], q, qt, k, kt)
            b.layer(l, kt, v, qt, ob)
            assert torch.equal(oa, ob) and not torch.equal(qt, q)


V = 40


class Drafted:
    """Two requests whose rows at a position are always the same, and so are what is drawn at a step and its rows; drafts of the target's likeliest tokens or of
    any."""

    def __init__(self, codes, seed=0, rows_of=(4, 6)):
        f, _ = rows.rope_frequencies(64)
        self.s = Session(codes=codes, vocab=V, rope=dict(rope_dims=64, rope_layout="half", rope_frequency=f), **SIZES)
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
        self.n = list(rows_of)
        self.q, self.k, self.v = (r(2, 2, 400, h, 64).bfloat16() for h in (8, 2, 2))  # [layer, request, position]
        self.target = torch.softmax(2.0 * r(2, 400, V), -1)  # [request, position]
        self.token = torch.where(r(2, 400) > -0.7, self.target.roll(1, 1).argmax(-1), torch.randint(0, V, (2, 400), device="cuda", generator=g)).int()
        self.draw, self.last = torch.rand(60, sum(self.n), device="cuda", generator=g), torch.rand(60, 2, device="cuda", generator=g)
        self.request = torch.tensor([0] * self.n[0] + [1] * self.n[1], device="cuda")
        self.out = torch.zeros(2, sum(self.n), 8, 64, device="cuda", dtype=torch.bfloat16)
        self.count = torch.zeros((), dtype=torch.long, device="cuda")
        self.log = torch.full((60, 2, 2), -7, dtype=torch.int32, device="cuda")
        self.threads = [self.s.open(i) for i in range(2)]

    def prompt(self, n0, n1):
        self.s.begin([self.threads[0]] * n0 + [self.threads[1]] * n1)
        at = torch.cat([torch.arange(n0), torch.arange(n1)]).cuda()
        of = torch.tensor([0] * n0 + [1] * n1).cuda()
        for l in range(2):
            self.s.layer(l, self.k[l, of, at], self.v[l, of, at], self.q[l, of, at], torch.empty(n0 + n1, 8, 64, device="cuda", dtype=torch.bfloat16))

    def body(self):
        """What a model would do of a step that has begun: nothing in it looks at the device's values."""
        at, i = self.s._step["position"].long().clone(), self.count
        for l in range(2):
            self.s.layer(l, self.k[l, self.request, at], self.v[l, self.request, at], self.q[l, self.request, at], self.out[l])
        acc, nxt = self.s.verify(self.token[self.request, at], self.target[self.request, at], self.draw.index_select(0, i.view(1))[0],
                                 self.last.index_select(0, i.view(1))[0])
        self.log.index_copy_(0, i.view(1), torch.stack([acc, nxt])[None])
        self.count += 1

    def contents(self):
        """K and V of both requests' tokens that are kept, [layer][request]."""
        s = self.s
        s._take_back()
        torch.cuda.synchronize()
        length, table, P = s.length.tolist(), s.page_table.cpu().numpy(), s.cfg.page_tokens
        out = []
        for l in range(2):
            for r in range(2):
                t = np.arange(length[r])
                slot = table[r, t // P] * P + t % P
                if s.cache is not None:
                    k, v = torch.zeros(2, len(t), 2, 64, device="cuda")
                    s.cache.read(l, torch.from_numpy(slot).int().cuda(), k, v)
                    torch.cuda.synchronize()
                    out.append((k, v))
        return length, out


def expected(d, steps, start):
    """(accepted, next token) of every step, positions after it, from the definition"""
    from test_gpu_rows_verify import one

    p, token, draw, last = d.target.double().cpu().numpy(), d.token.cpu().numpy(), d.draw.cpu().numpy(), d.last.cpu().numpy()
    at, log = list(start), []
    for i in range(steps):
        row, o = [], 0
        for r in range(2):
            n = d.n[r]
            span = slice(at[r], at[r] + n)
            row.append(one(p[r, span], None, token[r, span], draw[i, o:o + n], last[i, r], V))
            o += n
        log.append([[row[0][0], row[1][0]], [row[0][1], row[1][1]]])
        at = [a + 1 + x[0] for a, x in zip(at, row)]
    return np.array(log), at


@pytest.mark.parametrize("codes", ["e2m1", "int8"])
def test_drafts_step_by_step(codes):
    d = Drafted(codes)
    d.prompt(37, 5)
    for i in range(12):
        if i == 0 or i == 7:  # (anew from the host)
            if i:
                d.s.settle()
            d.s.begin([d.threads[0]] * d.n[0] + [d.threads[1]] * d.n[1])
        else:
            d.s.again()
        d.body()
        if i == 3:
            assert d.s.refused() == []
    want, at = expected(d, 12, (37, 5))
    assert np.array_equal(d.log[:12].cpu().numpy(), want) and 4 < want[:, 0].sum() < 12 * 8
    assert d.s.settle() == want[-1, 0].tolist() and [t.position for t in d.threads] == at
    length, got = d.contents()
    assert length == at
    if codes == "e2m1":  # what is kept is what a session without drafts writes
        plain = Drafted(codes)
        plain.prompt(*at)
        for a, b in zip(got, plain.contents()[1]):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("codes", ["e2m1", "e4m3"])
def test_drafts_replayed_from_a_graph(codes):
    a, b = Drafted(codes, 3), Drafted(codes, 3)
    stream = torch.cuda.Stream()
    for d in (a, b):
        d.prompt(20, 33)
        d.s.begin([d.threads[0]] * d.n[0] + [d.threads[1]] * d.n[1])
        d.body()
    for _ in range(11):
        b.s.again()
        b.body()
    torch.cuda.synchronize()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        a.s.bind(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            a.s.again()
            a.body()
        for i in range(11):
            graph.replay()
            if i % 4 == 1:  # the program's own work between replays
                torch.cuda.synchronize()
                (torch.ones(100, device="cuda") * i).sum().item()
    stream.synchronize()
    want, at = expected(a, 12, (20, 33))
    for d in (a, b):
        assert np.array_equal(d.log[:12].cpu().numpy(), want)
        assert d.s.settle() == want[-1, 0].tolist() and [t.position for t in d.threads] == at
    assert torch.equal(a.out, b.out)
    a.s.bind(torch.cuda.current_stream())
    (la, ca), (lb, cb) = a.contents(), b.contents()
    assert la == lb == at and int(a.s.free_count) == int(b.s.free_count)
    for x, y in zip(ca, cb):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_the_cache_fills_up_under_drafts():
    """A request that the cache has no room for is refused, keeps its tokens and its position, and goes on once there is room."""
    d = Drafted("e2m1", 5)
    d.s.release(0), d.s.release(1)
    s = d.s = Session(codes="e2m1", vocab=V, **{**SIZES, "n_phys_pages": 4})
    d.threads = [s.open(0), s.open(1)]
    d.prompt(30, 29)  # four pages
    s.begin([d.threads[0]] * 4 + [d.threads[1]] * 6)
    d.body()
    assert s.refused() == [0, 1] and s.accepted.tolist() == [0, 0] and s.next_token.tolist() == [-1, -1]
    s.settle()
    assert [t.position for t in d.threads] == [30, 29]
    s.again()
    torch.cuda.synchronize()
    assert s.length.tolist() == [30, 29]
    s.release(1)
    assert s.length.tolist() == [30, 0] and int(s.free_count) == 2
    s.begin([d.threads[0]] * 4)
    torch.cuda.synchronize()
    assert s.length.tolist() == [34, 0] and s._step["position"].tolist() == [30, 31, 32, 33]


def test_what_a_session_refuses_of_drafts():
    d = Drafted("e2m1", 6)
    s = d.s
    d.prompt(10, 10)
    kid = s.fork(d.threads[0])
    s.begin([d.threads[0], kid, d.threads[1]])
    with pytest.raises(ValueError):
        s.verify(None, None, None, None)  # two threads of a request
    s.join(d.threads[0], [kid])
    s.begin([d.threads[0]] * 4 + [d.threads[1]] * 6)
    d.body()
    for call in (lambda: s.begin([d.threads[0]]), lambda: s.fork(d.threads[0])):
        with pytest.raises(RuntimeError):
            call()
    s.settle()
    n = s.accepted.tolist()
    s.release(1)  # takes the drafts back
    assert s.length.tolist() == [11 + 1 + 1 + n[0], 0]


@pytest.mark.parametrize("seed", [7, 8, 9])
@pytest.mark.parametrize("verified", [False, True])
def test_another_request_goes_on_between_replays(verified, seed):
    """A captured step of one request, begun behind a verified one or not; the other request writes rows in between, and keeps them; each settle() finds the
    threads where the replays left them."""
    d = Drafted("e4m3", seed, rows_of=(4, 0))
    d.prompt(20, 33)
    one, other = d.threads
    stream = torch.cuda.Stream()
    d.s.begin([one] * 4)
    d.body()
    if not verified:  # four rows more that are kept, as the program says
        d.s.settle()
        d.s.begin([one] * 4, list(range(one.position, one.position + 4)))
        d.count += 1
    torch.cuda.synchronize()
    at = one.position if not verified else None
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        d.s.bind(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            d.s.again()
            d.body()
        rows_of_other, done = 33, 0
        for replays, more in ((1, 3), (2, 20), (1, 0), (2, 1)):
            for _ in range(replays):
                graph.replay()
            done += replays
            acc = d.s.settle()
            log = d.log[:int(d.count)].cpu().numpy()
            start = 20 + 1 + log[0, 0, 0] if verified else at
            first = 1 if verified else 2
            assert acc[0] == log[-1, 0, 0] and one.position == start + sum(1 + log[k, 0, 0] for k in range(first, first + done))
            assert other.position == rows_of_other
            if more:
                d.s.begin([other] * more)
                for l in range(2):
                    x = lambda h: torch.zeros(more, h, 64, device="cuda", dtype=torch.bfloat16)  # noqa: E731
                    d.s.layer(l, x(2), x(2), x(8), x(8))
                rows_of_other += more
                torch.cuda.synchronize()
                assert d.s.length.tolist()[1] == rows_of_other
    stream.synchronize()
    d.s._take_back()
    torch.cuda.synchronize()
    assert d.s.length.tolist() == [one.position, rows_of_other]
    print("accepted:", d.log[:int(d.count), 0, 0].tolist())


def test_a_release_between_a_verified_step_and_the_next():
    a, b = Drafted("e2m1", 8, rows_of=(4, 0)), Drafted("e2m1", 8, rows_of=(4, 0))
    for d in (a, b):
        d.prompt(20, 33)
        d.s.begin([d.threads[0]] * 4)
        d.body()
        if d is a:
            d.s.release(1)
        d.s.again()
        d.body()
        d.s.settle()
    assert torch.equal(a.log[:2, :, 0], b.log[:2, :, 0]) and a.threads[0].position == b.threads[0].position
    (la, ca), (lb, cb) = a.contents(), b.contents()
    assert la == [lb[0], 0] and lb[1] == 33
    for l in range(2):
        assert torch.equal(ca[2 * l][0], cb[2 * l][0]) and torch.equal(ca[2 * l][1], cb[2 * l][1])


def test_a_step_verified_twice_goes_by_the_second():
    a, b = Drafted("e2m1", 9), Drafted("e2m1", 9)
    for d in (a, b):
        d.prompt(20, 33)
        d.s.begin([d.threads[0]] * 4 + [d.threads[1]] * 6)
        if d is a:
            n = len(d.request)
            d.s.verify(torch.full((n,), -1, dtype=torch.int32, device="cuda"), d.target[0, :n], d.draw[0], d.last[0])  # (nothing is accepted)
        d.body()
        d.s.again()
        d.body()
        d.s.settle()
    assert torch.equal(a.log[:2], b.log[:2]) and [t.position for t in a.threads] == [t.position for t in b.threads]
    assert a.contents()[0] == b.contents()[0]


def test_a_session_without_a_vocabulary_verifies_nothing():
    s = Session(codes="e2m1", **SIZES)
    s.begin([s.open(0)])
    for call in (lambda: s.verify(None, None, None, None), s.settle):
        with pytest.raises(RuntimeError, match="vocab"):
            call()
    with pytest.raises(RuntimeError, match="begun"):
        Session(codes="e2m1", vocab=V, **SIZES).verify(None, None, None, None)
