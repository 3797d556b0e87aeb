"""Rows into the 8-bit cache for every number of rows that a work-group looks at (1, 2, 4, 8, 16), against the walk block by block: runs that begin on a
group's first and last row, go on past its end and past the next one's, rows without a slot between them, in handles for one request and for many."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_kv8_append import Cache, pytestmark, rows  # noqa: F401

SIZES = [(700, 1, 1), (500, 8, 2), (1600, 2, 2), (1200, 8, 4), (2500, 8, 8), (4200, 8, 16)]  # rows, kv heads, rows to a work-group (test_kv8_rules)


def runs(rng, n, group, blocks):
    """Slots of n rows: runs in blocks of their own, of every length and start, placed so that many begin at a group's last row or straddle groups."""
    order, slot = rng.permutation(blocks), []
    for i, b in enumerate(order):
        left = n - len(slot)
        if left <= 0:
            break
        kind = i % 6
        if kind == 0:  # up to a group's last row, without places
            slot += [-1] * ((group - 1 - len(slot)) % group)
        elif kind == 1:
            slot += [[-1, 1 << 30, -(1 << 31)][i % 3]]
        first = 0 if kind in (2, 3) else int(rng.integers(0, 16))
        many = 16 - first if kind in (0, 2) else int(rng.integers(1, 17 - first))
        slot += [int(b) * 16 + first + t for t in range(many)]
    assert len(slot) >= n
    return slot[:n]


@pytest.mark.parametrize("codes,D,dtype", [("e4m3", 64, "bf16"), ("int8", 128, "f16")])
@pytest.mark.parametrize("n,H,group", SIZES)
def test_runs_of_every_kind(n, H, group, codes, D, dtype):
    rng = np.random.default_rng([n, H, D])
    c = Cache(codes, H, D, 32, 360)
    for i in range(2):  # blocks that begin anew and blocks that go on
        c.append(runs(rng, n, group, 720), rows(i, n, H, D, dtype, 2.0), rows(10 + i, n, H, D, dtype, 2.0))
    c.check()


@pytest.mark.parametrize("n,H,group", SIZES[1:])
def test_a_prompt_and_the_rows_behind_it(n, H, group):
    """Rows of one request from the middle of a block on: a run begins on every 16th row, a group's first, last or in between."""
    c = Cache("e4m3", H, 64, 64, 200)
    table = np.random.default_rng(n).permutation(200)
    t = 0
    for i, m in enumerate((5, n, n)):
        at = np.arange(t, t + m)
        c.append(table[at // 64] * 64 + at % 64, rows(i, m, H, 64, "bf16"), rows(20 + i, m, H, 64, "bf16"))
        t += m
    c.check()


@pytest.mark.parametrize("n,H,group", SIZES)
def test_single_rows_of_as_many_blocks(n, H, group):
    c = Cache("int8", H, 64, 16, n)
    blocks = np.random.default_rng(n).permutation(n)
    c.append(blocks * 16 + np.arange(n) % 16, rows(1, n, H, 64, "f32"), rows(2, n, H, 64, "f32"))
    c.check()


def test_the_handles_capacity_changes_nothing():
    from paper_2502_11517_amd import kv8

    rng, n, H, D = np.random.default_rng(5), 4200, 8, 128
    slot = torch.tensor(runs(rng, n, 16, 720), dtype=torch.int32, device="cuda")
    x, y = rows(1, n, H, D, "bf16"), rows(2, n, H, D, "bf16")
    got = []
    for many in (1, 64, 4096):
        cfg = kv8.make_config("e4m3", "bf16", H, H, D, 1.0, max_rows=n, max_requests=many, page_tokens=32, n_phys_pages=360)
        k, v, ss = kv8.cache_shapes(cfg)
        b = [torch.zeros(s, dtype=t, device="cuda") for s, t in ((k, torch.uint8), (v, torch.uint8), (ss, torch.float32), (ss, torch.float32))]
        h = kv8.PastaKv8(cfg, torch.empty(kv8.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), k_codes=b[0], v_codes=b[1], k_scale=b[2],
                         v_scale=b[3], stream=torch.cuda.current_stream().cuda_stream)
        h.append(0, slot, x, y)
        torch.cuda.synchronize()
        got.append(b)
    assert all(torch.equal(p, q) for b in got[1:] for p, q in zip(got[0], b))
