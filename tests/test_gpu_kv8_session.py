"""The 8-bit cache's operators together: threads that fork and join, against attention over the rows that the fork history says are seen; steps
replayed from a graph against the same steps called."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv8_ref as ref
from paper_2502_11517_amd import kv8
from paper_2502_11517_amd.kv8_session import Session, main

pytestmark = pytest.mark.gpu


class Watched:
    """A session whose history is written down thread by thread: which rows (request's order) each thread's next row sees."""

    def __init__(self, seed, **kw):
        self.rng = np.random.default_rng(seed)
        torch.manual_seed(seed)
        self.kw = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, softmax_scale=0.125, max_requests=3, max_rows=256, n_phys_pages=200, pages_per_request=60)
        self.kw.update(kw)
        self.s = Session(**self.kw)
        self.seen = {}  # id(thread) -> rows seen
        self.rows = [0] * 3
        self.k, self.v = ([[] for _ in range(3)] for _ in range(2))

    def open(self, r):
        t = self.s.open(r)
        self.seen[id(t)] = []
        return t

    def fork(self, p, **kw):
        t = self.s.fork(p, **kw)
        self.seen[id(t)] = list(self.seen[id(p)])
        return t

    def join(self, t, others):
        self.s.join(t, others)
        self.seen[id(t)] = sorted(set(self.seen[id(t)]).union(*(self.seen[id(o)] for o in others)))

    def step(self, rows, check=True):
        s, n = self.s, len(rows)
        c = s.cfg
        td = {kv8.BF16: torch.bfloat16, kv8.F16: torch.float16}[c.dtype]
        x = lambda h: torch.randn(n, h, c.head_dim, device="cuda").to(td)  # noqa: E731
        q, k, v = x(c.n_q_heads), x(c.n_kv_heads), x(c.n_kv_heads)
        out, lse = torch.empty_like(q), torch.empty(n, c.n_q_heads, device="cuda")
        s.begin(rows)
        s.layer(0, k, v, q, out, lse)
        torch.cuda.synchronize()
        kc, vc = self.values()
        slot, table = s.slot.cpu().numpy(), s.page_table.cpu().numpy()
        P, G = c.page_tokens, c.n_q_heads // c.n_kv_heads
        for i, t in enumerate(rows):
            self.seen[id(t)].append(self.rows[t.request])
            self.rows[t.request] += 1
            j = np.array(self.seen[id(t)])
            at = table[t.request, j // P] * P + j % P
            assert at[-1] == slot[i]
            if not check or i % 7:
                continue
            for h in range(c.n_q_heads):
                z = kc[at, h // G] @ q[i, h].double().cpu().numpy() * c.softmax_scale
                m = z.max()
                w = np.exp(z - m)
                want = w @ vc[at, h // G] / w.sum()
                tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * (w @ np.abs(vc[at, h // G])) / w.sum() + len(at) * 2.0 ** -25 * np.abs(vc[at, h // G]).max()
                assert (np.abs(out[i, h].double().cpu().numpy() - want) <= tol).all()
                assert abs(float(lse[i, h]) - (m + np.log(w.sum()))) <= 2.0 ** -18 * (1 + abs(m))
        assert self.s.length.cpu().tolist() == self.rows

    def values(self):
        s, val = self.s, ref.code_values({kv8.E4M3: "e4m3", kv8.INT8: "int8"}[self.s.cfg.codes])
        out = []
        for codes, scale, keys in ((s.k_codes, s.k_scale, True), (s.v_codes, s.v_scale, False)):
            b = codes[0].cpu().numpy()
            x = val[ref.k_natural(b) if keys else np.moveaxis(b, -1, -2)] * scale[0].cpu().numpy()[..., None, None]
            out.append(x.transpose(0, 2, 3, 1, 4).reshape(-1, s.cfg.n_kv_heads, s.cfg.head_dim))
        return out


@pytest.mark.parametrize("codes,dtype,seed", [("e4m3", "bf16", 1), ("int8", "bf16", 2), ("e4m3", "f16", 3)])
def test_random_forks_and_joins(codes, dtype, seed):
    w = Watched(seed, codes=codes, dtype=dtype)
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
        rows = [t for r in range(3) for t in live[r] if rng.random() < 0.8]
        if rows:
            w.step(rows)


def test_tags_run_out_and_are_free_again_after_the_join():
    w = Watched(4)
    root = w.open(0)
    w.step([root] * 5)
    kids = []
    with pytest.raises(RuntimeError):
        for _ in range(40):
            kids.append(w.fork(root))
    assert len(kids) == 31
    w.step(kids)
    w.join(root, kids)
    w.step([root] * 3)
    w.step([w.fork(root), root])


def test_a_released_requests_pages_come_back():
    w = Watched(5)
    a, b = w.open(0), w.open(1)
    w.step([a] * 100 + [b] * 20)
    left = int(w.s.free_count)
    w.s.release(0)
    w.rows[0] = 0
    w.step([b])
    assert int(w.s.free_count) == left + 7 and w.s.length.cpu().tolist()[:2] == [0, 21]
    w.step([w.open(0)] * 30)


def test_a_full_cache_refuses_a_request_and_its_rows_see_nothing():
    s = Session(n_q_heads=2, n_kv_heads=2, head_dim=64, softmax_scale=0.125, max_requests=2, max_rows=64, n_phys_pages=3, pages_per_request=8)
    a, b = s.open(0), s.open(1)
    x = lambda n, h: torch.randn(n, h, 64, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    s.begin([a] * 20 + [b] * 30)
    out, lse = torch.full((50, 2, 64), 7.0, device="cuda", dtype=torch.bfloat16), torch.zeros(50, 2, device="cuda")
    s.layer(0, x(50, 2), x(50, 2), x(50, 2), out, lse)
    torch.cuda.synchronize()
    assert s.length.tolist() == [20, 0] and int(s.free_count) == 1 and (s.slot[20:50] == -1).all()
    assert (out[20:] == 0).all() and torch.isneginf(lse[20:]).all() and torch.isfinite(lse[:20]).all()


@pytest.mark.parametrize("n", [3, 40])
def test_replays_of_one_captured_step_are_the_steps_called(n):
    """Thirty replays, with eager work and synchronisation between them, each against the eager session; single rows, and more than a wave's."""
    sessions, outs = [], []
    for captured in (False, True):
        torch.manual_seed(9)
        s = Session(n_q_heads=8, n_kv_heads=2, head_dim=128, softmax_scale=0.09, n_layers=2, max_rows=128, n_phys_pages=400, pages_per_request=300,
                    slopes=[0.01 * i for i in range(8)], logit_cap=30.0)
        root = s.open(0)
        data = [[torch.randn(m, h, 128, device="cuda").bfloat16() for h in (8, 2, 2)] for m in [100, n] + [n] * 30]
        q, k, v = (torch.empty_like(x) for x in data[1])
        out, lse = torch.zeros_like(q), torch.zeros(n, 8, device="cuda")

        def forward(a, b, c, o, e=None):
            for l in range(2):
                s.layer(l, b, c, a, o, e)

        s.begin([root] * 100)
        forward(*data[0], torch.empty_like(data[0][0]))
        threads = [s.fork(root) for _ in range(min(n, 31))]
        threads = (threads * 2)[:n]
        s.begin(threads)
        s._step["position"].add_(1)
        for x, y in zip((q, k, v), data[1]):
            x.copy_(y)
        forward(q, k, v, out, lse)
        torch.cuda.synchronize()
        got = [(out.clone(), lse.clone())]
        if captured:
            stream = torch.cuda.Stream()
            step = s._step
            s.bind(stream)
            s._step = step
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                s.again()
                forward(q, k, v, out, lse)
        for i in range(30):
            for x, y in zip((q, k, v), data[2 + i]):
                x.copy_(y)
            torch.cuda.synchronize()
            if captured:
                g.replay()
            else:
                s.again()
                forward(q, k, v, out, lse)
            torch.cuda.synchronize()
            got.append((out.clone(), lse.clone()))
            (torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()
        sessions.append(s), outs.append(got)
    a, b = sessions
    for (x, y), (z, w) in zip(*outs):
        assert torch.equal(x, z) and torch.equal(y, w)
    pages = a.page_table[0, :-(-int(a.length[0]) // 16)].long()
    assert torch.equal(a.length, b.length) and torch.equal(a.page_table, b.page_table) and torch.equal(a.free_count, b.free_count)
    assert torch.equal(a.k_scale[:, pages], b.k_scale[:, pages]) and int(a.length[0]) == 100 + n * 31


@pytest.mark.parametrize("twice", [False, True])
def test_going_on_is_the_same_as_beginning_again(twice):
    """again() against begin() with the same threads: places, positions (and so the scores, which distance lowers), outputs."""
    got = []
    for begin in (True, False):
        torch.manual_seed(11)
        s = Session(n_q_heads=4, n_kv_heads=2, head_dim=64, softmax_scale=0.125, max_rows=64, n_phys_pages=60, pages_per_request=40,
                    slopes=[0.5, 0.25, 0.125, 0.0625])
        root = s.open(0)
        x = lambda n, h: torch.randn(n, h, 64, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        s.begin([root] * 20)
        s.layer(0, x(20, 2), x(20, 2), x(20, 4), torch.empty(20, 4, 64, device="cuda", dtype=torch.bfloat16))
        threads = [s.fork(root) for _ in range(3)] * (2 if twice else 1)
        threads.sort(key=id)
        n = len(threads)
        for i in range(5):
            if begin or i == 0:
                s.begin(threads)
            else:
                s.again()
                s.advanced(threads, 1)
            out, lse = torch.empty(n, 4, 64, device="cuda", dtype=torch.bfloat16), torch.empty(n, 4, device="cuda")
            s.layer(0, x(n, 2), x(n, 2), x(n, 4), out, lse)
            got.append((out, lse, s.slot[:n].clone(), s.slot_position[s.slot[:n].long()]))
        assert sorted(t.position for t in threads) == [20 + 5 * n // 3] * n
    for a, b in zip(got[:5], got[5:]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_what_a_released_request_held_is_not_seen_by_the_next_one_even_if_that_is_refused():
    s = Session(n_q_heads=2, n_kv_heads=2, head_dim=64, softmax_scale=0.125, max_requests=2, max_rows=64, n_phys_pages=4, pages_per_request=8)
    x = lambda n, h: torch.randn(n, h, 64, device="cuda", dtype=torch.bfloat16)  # noqa: E731

    def step(rows):
        n = len(rows)
        out, lse = torch.empty(n, 2, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(n, 2, device="cuda")
        s.begin(rows)
        s.layer(0, x(n, 2), x(n, 2), x(n, 2), out, lse)
        return out, lse

    a, b = s.open(0), s.open(1)
    step([a] * 32 + [b] * 16)
    s.release(0)
    assert s.length.tolist() == [0, 16] and int(s.free_count) == 3
    a = s.open(0)
    out, lse = step([a] * 60)  # four pages
    assert s.length.tolist() == [0, 16] and (out == 0).all() and torch.isneginf(lse).all()
    kid = s.fork(a)
    step([a] * 5 + [kid] * 3)
    s.join(a, [kid])
    assert s.prefix_len.tolist() == [8, 0] == [int(s.length[0]), 0]
    step([a])
    assert s.length.tolist() == [9, 16]


def test_the_example_runs(capsys):
    main()
    assert "tokens 400" in capsys.readouterr().out
