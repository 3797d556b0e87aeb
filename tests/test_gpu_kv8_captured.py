"""A captured step among others: replays with steps of another request, and memory that is taken and overwritten, between them, against the same steps
called one by one (equal: the kernels do the same work)."""
from __future__ import annotations

import pytest
import torch

from paper_2502_11517_amd.kv8_session import Session

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [3, 40])
def test_a_captured_step_keeps_its_rows_when_others_are_begun(n):
    runs = []
    for captured in (False, True):
        torch.manual_seed(21)
        s = Session(n_q_heads=8, n_kv_heads=2, head_dim=64, softmax_scale=0.125, n_layers=2, max_requests=2, max_rows=128, n_phys_pages=300,
                    pages_per_request=150, slopes=[0.01 * i for i in range(8)])
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        got = []
        with torch.cuda.stream(stream):
            x = lambda m, h: torch.randn(2, m, h, 64, device="cuda", dtype=torch.bfloat16)  # noqa: E731

            def forward(q, k, v, out, lse):
                for l in range(2):
                    s.layer(l, k[l], v[l], q[l], out[l], lse[l])

            def other(rows):  # a step of the other request; what it leaves on the device is overwritten behind it
                s.begin(rows)
                m = len(rows)
                out, lse = torch.empty(2, m, 8, 64, device="cuda", dtype=torch.bfloat16), torch.empty(2, m, 8, device="cuda")
                forward(x(m, 8), x(m, 2), x(m, 2), out, lse)
                got.append((out.clone(), lse.clone()))
                for size in (n, 4 * n, 8 * n, 64, 1024):
                    for _ in range(8):
                        torch.full((size,), -1, dtype=torch.uint8, device="cuda")

            s.bind(stream)
            root, alone = s.open(0), s.open(1)
            other([root] * 60)
            threads = [s.fork(root) for _ in range(min(n, 31))]
            threads = (threads * 2)[:n]
            q, k, v = x(n, 8), x(n, 2), x(n, 2)
            out, lse = torch.empty_like(q), torch.empty(2, n, 8, device="cuda")
            other(threads)
            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    s.again()
                    forward(q, k, v, out, lse)
            for i in range(12):
                q.copy_(x(n, 8)), k.copy_(x(n, 2)), v.copy_(x(n, 2))
                if captured:
                    graph.replay()
                    s.advanced(threads, 1)
                else:
                    s.begin(threads)
                    forward(q, k, v, out, lse)
                got.append((out.clone(), lse.clone()))
                if i % 3 == 1:
                    other([alone] * (1 + 9 * i))
                if i % 4 == 3:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        runs.append((s, got, [t.position for t in threads]))
    (a, x, p), (b, y, r) = runs
    assert len(x) == len(y) and p == r
    for (o, e), (w, f) in zip(x, y):
        assert torch.equal(o, w) and torch.equal(e, f)
    assert torch.equal(a.length, b.length) and torch.equal(a.page_table, b.page_table) and a.length.tolist() == [60 + 13 * n, 4 + 9 * (1 + 4 + 7 + 10)]


def test_a_refused_requests_rows_take_the_same_ids_when_there_is_room():
    """Against a session that had the room from the start: places differ, positions and so the scores, which distance lowers, do not."""
    runs = []
    for pages in (5, 9):
        torch.manual_seed(3)
        s = Session(n_q_heads=2, n_kv_heads=2, head_dim=64, softmax_scale=0.125, max_requests=2, max_rows=128, n_phys_pages=pages, pages_per_request=8,
                    slopes=[0.5, 0.125])
        x = lambda n, h: torch.randn(n, h, 64, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        a, b = s.open(0), s.open(1)

        def step(rows):
            s.begin(rows)
            out, lse = torch.empty(len(rows), 2, 64, device="cuda", dtype=torch.bfloat16), torch.empty(len(rows), 2, device="cuda")
            s.layer(0, x(len(rows), 2), x(len(rows), 2), x(len(rows), 2), out, lse)
            return out, lse

        step([a] * 48 + [b] * 20)
        assert s.refused() == []
        if pages == 5:
            out, lse = step([b] * 30)
            assert s.refused() == [1] and b.position == 20 and s.length.tolist() == [48, 20] and torch.isneginf(lse).all()
            torch.manual_seed(4)
            s.release(0)
        torch.manual_seed(4)
        runs.append(step([b] * 30))
        assert s.refused() == [] and b.position == 50 and int(s.length[1]) == 50
        runs.append(step([b]))
    assert all(torch.equal(x, y) for i in (0, 1) for x, y in zip(runs[i], runs[i + 2]))
