"""Rows whose ascending slots leave out others of a block: what is in those stays, and no row's codes are lost, however many rows a work-group takes."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_kv4_rows import Cache, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("slot", [[3, 5], [0, 15], [1, 14, 15], [0, 2, 3, 6], list(range(0, 16, 2)), list(range(1, 16, 2)), [t for t in range(16) if t != 7],
                                  [3, 5, 16, 18, 31, 33], [14, 15, 17, 18], [9, -1, 16, 18, 1 << 20, 35, 37], [40, 42, 8, 10]], ids=str)
def test_slots_left_out(slot, D, dtype):
    c = Cache(3, D, 32, 2, seed=D)
    c.append(slot, rows(1, len(slot), 3, D, dtype), rows(2, len(slot), 3, D, dtype))
    c.check()


@pytest.mark.parametrize("n", [40, 350, 700, 1700, 4300])
def test_any_subsets_of_blocks(n):
    """Rows of random subsets of the blocks, in any order of the blocks: one, two, four, eight and sixteen rows to a work-group."""
    rng = np.random.default_rng(n)
    H, D, P = 8, 64, 32
    pages = n // 8
    slot = []
    for b in rng.permutation(pages * P // 16):
        k = int(rng.choice([1, 2, 3, 8, 13, 15, 16]))
        slot += [int(b) * 16 + int(t) for t in np.sort(rng.permutation(16)[:k])]
        if rng.random() < 0.2:
            slot.append(-1)
    assert len(slot) >= n
    c = Cache(H, D, P, pages, seed=n)
    c.append(slot[:n], rows(1, n, H, D, "bf16"), rows(2, n, H, D, "bf16"))
    c.check()


def test_gaps_are_filled_later():
    c = Cache(2, 128, 16, 3)
    for i, slot in enumerate(([0, 4, 9, 20, 22], [1, 2, 3, 5, 21], [6, 8, 10, 15, 16, 47], [7, 11, 12, 13, 14])):
        c.append(slot, rows(i, len(slot), 2, 128, "bf16"), rows(9 + i, len(slot), 2, 128, "bf16"))
        c.check()
