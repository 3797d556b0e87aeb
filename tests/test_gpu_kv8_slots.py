"""Places of a step's rows against the walk request by request (whole numbers: equal)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv8_ref as ref
from paper_2502_11517_amd import kv8

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.int32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


class Step:
    def __init__(self, rng, R, P, W, length, keep, rows, slack, pad=0, meta=True):
        self.R, self.P, self.W, self.length, self.keep = R, P, W, np.asarray(length), keep
        self.offs = np.concatenate([[0], np.cumsum(rows)]).astype(int)
        self.n = int(self.offs[-1]) + pad
        need = [-(-int(x) // P) for x in length]
        self.pages = sum(need) + slack
        perm = rng.permutation(self.pages)
        self.table = np.full((R, W), -1)
        at = 0
        for r, k in enumerate(need):
            self.table[r, :k] = perm[at:at + k]
            at += k
        self.free = slack
        self.stack = np.concatenate([perm[at:], np.full(self.pages - slack, -5)])
        self.tag = rng.integers(0, 64, self.n) if meta else None
        self.pos = rng.integers(0, 1 << 20, self.n) if meta else None

    def run(self, in_place=False, n_requests=None):
        P = self.P
        cfg = kv8.make_config("e4m3", "bf16", 4, 1, 64, 1.0, max_requests=max(1, self.R), max_rows=max(1, self.n), page_tokens=P,
                              n_phys_pages=max(1, self.pages), pages_per_request=self.W)
        d = dict(table=dev(self.table), stack=dev(self.stack), tag=torch.full((self.pages * P + 16,), 255, dtype=torch.uint8, device="cuda"),
                 pos=torch.full((self.pages * P + 16,), -1, dtype=torch.int32, device="cuda"), length=dev(self.length), free=dev([self.free]),
                 slot=torch.full((max(1, self.n),), -77, dtype=torch.int32, device="cuda"))
        d["length_out"] = d["length"] if in_place else torch.full_like(d["length"], -3)
        d["free_out"] = d["free"] if in_place else torch.full_like(d["free"], -3)
        h = kv8.PastaKv8(cfg, torch.empty(kv8.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), page_table=d["table"],
                         free_pages=d["stack"], slot_tag=d["tag"], slot_position=d["pos"], stream=torch.cuda.current_stream().cuda_stream)
        h.slots(d["length"], dev(self.offs), self.n, d["slot"], d["length_out"], d["free"], d["free_out"], keep=dev(self.keep),
                row_tag=dev(self.tag, torch.uint8), row_position=dev(self.pos))
        torch.cuda.synchronize()
        return {k: v.cpu().numpy() for k, v in d.items()}

    def check(self, **kw):
        slot, out, free, table, stack = ref.slots(self.P, self.W, self.length, self.keep, self.offs, self.n, self.table, self.stack, self.free)
        got = self.run(**kw)
        assert np.array_equal(got["slot"][:self.n], slot)
        assert np.array_equal(got["length_out"], out) and got["free_out"][0] == free
        assert np.array_equal(got["table"], table) and np.array_equal(got["stack"], stack)
        good = slot >= 0
        assert len(np.unique(slot[good])) == good.sum()
        if self.tag is not None:
            tag, pos = np.full(len(got["tag"]), 255), np.full(len(got["pos"]), -1)
            tag[slot[good]], pos[slot[good]] = self.tag[good], self.pos[good]
            assert np.array_equal(got["tag"], tag) and np.array_equal(got["pos"], pos)
        return slot, out


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("R,most,rows", [(1, 0, 1), (1, 100, 1), (1, 0, 300), (16, 300, 8), (64, 40, 3), (65, 40, 3), (200, 200, 20), (256, 30, 40), (257, 90, 3), (512, 60, 5),
                                         (700, 60, 5), (1024, 50, 3), (1025, 50, 3), (1500, 90, 5),
                                         (3, 50, 3000), (3, 50, 6000)])
def test_steps_of_all_sizes(P, R, most, rows):
    rng = np.random.default_rng([P, R, rows])
    length = rng.integers(0, most + 1, R)
    new = rng.integers(0, rows + 1, R)
    new[0] = rows
    need = int((-(-(length + new) // P) - -(-length // P)).sum())
    Step(rng, R, P, -(-(most + rows) // P), length, None, new, need + 3, pad=R % 3).check()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("R", [7, 90, 400, 1000, 1100])
def test_rows_taken_back_and_requests_released(R, in_place):
    rng = np.random.default_rng(R)
    P = 16
    length = rng.integers(0, 400, R)
    keep = np.where(rng.random(R) < 0.5, np.maximum(0, length - rng.integers(0, 60, R)), length + rng.integers(0, 5, R))
    gone = rng.random(R) < 0.2
    keep = np.where(gone, 0, keep)
    new = np.where(gone, 0, rng.integers(0, 40, R))
    Step(rng, R, P, 64, length, keep, new, 2 * R + 10, meta=False).check(in_place=in_place)


@pytest.mark.parametrize("R,slack", [(5, 0), (12, 3), (100, 40), (1300, 500)])
def test_requests_that_the_stack_cannot_serve_change_nothing(R, slack):
    rng = np.random.default_rng([R, slack])
    length = rng.integers(0, 100, R)
    slot, out = Step(rng, R, 16, 16, length, None, rng.integers(0, 30, R), slack).check()
    assert (out == length).sum() > 0 and (slot < 0).any()


def test_a_request_that_would_outgrow_its_table_is_refused_and_counts_for_nobody():
    rng = np.random.default_rng(1)
    s = Step(rng, 4, 16, 4, [60, 64, 10, 0], None, [4, 1, 54, 65], 8)
    slot, out = s.check()
    assert out.tolist() == [64, 64, 64, 0]


def test_pages_given_back_are_taken_in_the_same_step():
    rng = np.random.default_rng(2)
    s = Step(rng, 3, 16, 8, [100, 0, 33], [0, 0, 33], [0, 96, 16], 0)
    _, out = s.check()
    assert out.tolist() == [0, 96, 49]  # seven pages came back, seven were needed


def test_no_rows_and_no_requests():
    rng = np.random.default_rng(3)
    Step(rng, 3, 16, 4, [3, 0, 20], None, [0, 0, 0], 2).check()
    Step(rng, 3, 16, 4, [3, 0, 20], [1, 0, 3], [0, 0, 0], 2, pad=5).check()


def test_bad_page_numbers_and_lengths_stay_inside_the_arrays():
    rng = np.random.default_rng(4)
    s = Step(rng, 4, 16, 4, [5, 20, 7, 3], None, [2, 2, 20, 1], 6)
    s.table[0, 0], s.table[1, 1] = -1, 1 << 30
    s.stack[:6] = [-1, 1 << 28, s.pages, -1 << 31, -7, s.pages + 1]
    got = s.run()
    assert got["slot"][:4].tolist() == [-1] * 4 and (got["slot"][13:24] == -1).all()  # bad pages, old and new, have no slots
    assert got["slot"][4:13].tolist() == [s.table[2, 0] * 16 + 7 + i for i in range(9)] and got["slot"][24] == s.table[3, 0] * 16 + 3
    s.length = np.array([1 << 30, -5, 7, 3])
    s.free = 1 << 30
    s.run()
