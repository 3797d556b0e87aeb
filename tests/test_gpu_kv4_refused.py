"""A step that the cache has no room for behind one whose drafts were rejected: tokens, positions and outputs go on as if it had not been, called and replayed, by the
session and by the C ABI alone."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2502_11517_amd import kv8, rows
from paper_2502_11517_amd.kv8_session import Session
from test_gpu_kv4_session import SIZES, V, Drafted
from test_gpu_rows_verify import one

pytestmark = pytest.mark.gpu


def drafted(codes, pages, seed):
    """One request of five rows a step, of whose first drafts two are accepted, and another that holds a page."""
    d = Drafted(codes, seed, rows_of=(5, 0))
    f, _ = rows.rope_frequencies(64)
    d.s = Session(codes=codes, vocab=V, rope=dict(rope_dims=64, rope_layout="half", rope_frequency=f), **{**SIZES, "n_phys_pages": pages})
    d.threads = [d.s.open(0), d.s.open(1)]
    d.draw[0] = torch.tensor([0.0, 0.0, 0.0, 1.0, 1.0])
    d.target.clamp_(min=1e-6)  # (a draw of 0 is below every probability, one of 1 below none)
    d.prompt(27, 16)
    d.s.begin([d.threads[0]] * 5)
    d.body()
    return d


@pytest.mark.parametrize("how", ["again", "begin", "replayed"])
@pytest.mark.parametrize("codes", ["e2m1", "e4m3", "int8"])
def test_a_refused_step_behind_a_verified_one(codes, how):
    a, b = drafted(codes, 3, 1), drafted(codes, 60, 1)  # 32 tokens of which 30 are kept, and no page left; room for all
    outs = {id(a): [], id(b): []}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def go_on(d):
        if how == "replayed":
            d.graph.replay()
            stream.synchronize()
        elif how == "again":
            d.s.again()
            d.body()
        else:
            d.s.settle()
            d.s.begin([d.threads[0]] * 5)
            d.body()
        outs[id(d)].append(d.out.clone())

    with torch.cuda.stream(stream if how == "replayed" else torch.cuda.current_stream()):
        if how == "replayed":
            for d in (a, b):
                d.s.bind(stream)
                d.graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(d.graph, stream=stream):
                    d.s.again()
                    d.body()
        for _ in range(2):
            go_on(a)
            torch.cuda.synchronize()
            assert a.s.accepted.tolist() == [0, 0] and a.s.next_token.tolist() == [-1, -1] and a.s.length.tolist() == [30, 16]
        b.count += 2  # (what is drawn in these steps)
        for d in (a, b):
            d.s.release(1)
            for _ in range(6):
                go_on(d)
    torch.cuda.synchronize()
    log = [d.log[:9].cpu().numpy() for d in (a, b)]
    assert log[0][0, 0, 0] == 2 and (log[0][1:3, :, 0] == [0, -1]).all() and np.array_equal(log[0][3:, :, 0], log[1][3:, :, 0])
    p, token, draw, last = b.target[0].double().cpu().numpy(), b.token[0].cpu().numpy(), b.draw.cpu().numpy(), b.last[:, 0].cpu().numpy()
    at = 27
    for i in (0, *range(3, 9)):  # from the definition, with the draws of the step
        want = one(p[at:at + 5], None, token[at:at + 5], draw[i], last[i], V)
        assert log[0][i, :, 0].tolist() == list(want)
        at += 1 + want[0]
    for x, y in zip(outs[id(a)][2:], outs[id(b)]):
        assert torch.equal(x, y)
    for d in (a, b):
        d.s.settle()
    assert a.threads[0].position == b.threads[0].position == at > 30
    (la, ca), (lb, cb) = a.contents(), b.contents()
    assert la == lb == [at, 0]
    for x, y in zip(ca, cb):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


@pytest.mark.parametrize("replayed", [False, True])
def test_the_loop_of_slots_and_verify_alone(replayed):
    """Drafts taken back by a call without rows, then the step's places, then verify, in place: a refused step between them changes nothing."""
    i32 = dict(dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream() if replayed else torch.cuda.current_stream()
    cfg = kv8.make_config("e4m3", "bf16", 4, 1, 64, 1.0, max_requests=2, max_rows=64, page_tokens=16, n_phys_pages=3, pages_per_request=30)
    length, free, slot, keep = torch.tensor([32, 16], **i32), torch.tensor([0], **i32), torch.full((5,), -1, **i32), torch.tensor([30, 16], **i32)
    table = torch.full((2, 30), -1, **i32)
    table[0, 0], table[0, 1], table[1, 0] = 0, 1, 2
    h = kv8.PastaKv8(cfg, torch.empty(kv8.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), page_table=table, free_pages=torch.zeros(3, **i32),
                     stream=stream.cuda_stream)
    rcfg = rows.make_config(vocab=V, max_sequences=2, max_rows=5)
    r = rows.PastaRows(rcfg, torch.empty(rows.query_workspace_bytes(rcfg), dtype=torch.uint8, device="cuda"), stream=stream.cuda_stream)
    offs, none = torch.tensor([0, 5, 5], **i32), torch.zeros(3, **i32)
    target, token = torch.full((5, V), 1.0 / V, device="cuda"), torch.zeros(5, **i32)
    draw, last = torch.tensor([0.0, 0.0, 0.0, 1.0, 1.0], device="cuda"), torch.zeros(2, device="cuda")
    acc, nxt, pos = torch.zeros(2, **i32), torch.zeros(2, **i32), torch.arange(30, 35, **i32)
    torch.cuda.synchronize()

    def step():
        h.slots(length, none, 0, None, length, free, free, keep=keep)
        h.slots(length, offs, 5, slot, length, free, free)
        r.verify(offs, token, target, draw, last, acc, nxt, length=length, keep=keep, row_position=pos, position_out=pos, slot=slot)

    go = step
    if replayed:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        go = graph.replay
    for _ in range(3):
        go()
        torch.cuda.synchronize()
        assert length.tolist() == [30, 16] and keep.tolist() == [30, 16] and acc.tolist() == [0, 0] and pos.tolist() == list(range(30, 35))
    h.slots(length, none, 0, None, length, free, free, keep=torch.tensor([30, 0], **i32))  # the other request's page comes back
    for i in range(1, 4):  # each step keeps three of five rows
        torch.cuda.synchronize()
        go()
        torch.cuda.synchronize()
        at = 30 + 3 * i
        assert length.tolist() == [at + 2, 0] and keep.tolist() == [at, 0] and acc.tolist() == [2, 0] and pos.tolist() == list(range(at, at + 5))
        assert slot.tolist() == [int(table[0, t // 16]) * 16 + t % 16 for t in range(at - 3, at + 2)]
