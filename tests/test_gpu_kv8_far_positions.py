"""Scores lowered by distance where positions take all of 32 bits: no distance up to 2^32 - 1 wraps.  Bounds are those of test_gpu_kv8_attend; distances
themselves are rounded to fp32 once, which its 2^-20 of the largest score covers."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_kv8_attend import SHAPES, Case, pytestmark  # noqa: F401

LOW, HIGH = -(1 << 31), (1 << 31) - 1


@pytest.mark.parametrize("codes,dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("ordered", [False, True])
def test_positions_at_both_ends(codes, dtype, D, Hq, Hkv, n, ordered):
    """Rows at both ends and between, blocks whose positions ascend (from both ends, and over the end of the whole numbers) or lie anywhere."""
    c = Case([n, D], codes, dtype, Hq, Hkv, D, 16, [500], [n])
    t = np.arange(500)
    pos = c.rng.integers(LOW, HIGH + 1, 500)
    if ordered:
        start = np.array([LOW, HIGH - 15, -8, 5, HIGH - 500, LOW + 100])[t // 16 % 6]
        pos = start + t % 16
        over = t // 16 % 7 == 6
        pos[over] = (HIGH - 7 + t[over] % 16 + (1 << 31)) % (1 << 32) - (1 << 31)  # HIGH - 7 ... HIGH, LOW ... LOW + 7
    c.position[c.table[0, t // 16] * 16 + t % 16] = pos
    row = c.rng.integers(LOW, HIGH + 1, n)
    row[:4] = LOW, HIGH, 0, HIGH - 3
    c.check(slopes=c.rng.uniform(0.2e-9, 2e-9, Hq).astype(np.float32), row_position=row)
