"""What an 8-bit cache holds behind drafts that a session takes back in replays."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv8_ref as ref
from paper_2502_11517_amd import kv8
from test_gpu_kv4_session import SIZES, Drafted

pytestmark = pytest.mark.gpu


def held(s):
    """(lengths; K and V of every request's kept tokens, layer by layer) of an 8-bit session, as its codes and scales say."""
    s._take_back()
    torch.cuda.synchronize()
    values, P = ref.code_values({kv8.E4M3: "e4m3", kv8.INT8: "int8"}[s.cfg.codes]), s.cfg.page_tokens
    length, table, out = s.length.tolist(), s.page_table.cpu().numpy(), []
    for l in range(s.cfg.n_layers):
        for codes, scale, keys in ((s.k_codes, s.k_scale, True), (s.v_codes, s.v_scale, False)):
            b = codes[l].cpu().numpy()
            x = values[ref.k_natural(b) if keys else np.moveaxis(b, -1, -2)] * scale[l].cpu().numpy()[..., None, None]
            x = x.transpose(0, 2, 3, 1, 4).reshape(-1, s.cfg.n_kv_heads, s.cfg.head_dim)
            for r, n in enumerate(length):
                t = np.arange(n)
                out.append(x[table[r, t // P] * P + t % P])
    return length, out


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_what_an_8_bit_cache_holds_behind_replayed_drafts(codes):
    a, b = Drafted(codes, 3), Drafted(codes, 3)
    stream = torch.cuda.Stream()
    for d in (a, b):
        d.prompt(20, 33)
        d.s.begin([d.threads[0]] * d.n[0] + [d.threads[1]] * d.n[1])
        d.body()
    for _ in range(9):
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
        for _ in range(9):
            graph.replay()
    stream.synchronize()
    a.s.bind(torch.cuda.current_stream())
    (la, ca), (lb, cb) = held(a.s), held(b.s)
    assert la == lb and len(ca) == len(cb) == 8 and all(len(x) > 30 for x in ca)
    for x, y in zip(ca, cb):
        assert np.array_equal(x, y) and np.isfinite(x).all() and (x != 0).mean() > 0.5
    # and it is the rows that were accepted: V goes in as it is, to half a step of e4m3 (2^-4, or that of its smallest numbers), or less than a step of 2^e int8, of which
    # 127 are half of the block's largest value or more (all are below 8 here)
    v = a.v.double().cpu().numpy()
    for l in range(2):
        for r in range(2):
            want = v[l, r, :la[r]]
            step = {"e4m3": 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * 8 / 448, "int8": np.full_like(want, 2 * 8 / 127)}[codes]
            assert (np.abs(ca[4 * l + 2 + r] - want) <= step + 1e-9).all()
