"""Attention over the 4-bit cache where its plan changes: tokens on both sides of every rule by which tiles are split, requests that fill the chip
exactly or by one tile more, positions in order, pieces joined from few parts and from many.  Bounds are those of test_gpu_kv4_attend."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_kv4_attend import SHAPES, Case, pytestmark  # noqa: F401


@pytest.mark.parametrize("n", [1, 5, 33])
@pytest.mark.parametrize("T", [127, 129, 255, 257, 384, 385, 511, 513, 640, 767, 768, 769, 1024, 1025, 1153, 2047, 4099])
def test_tokens_around_the_lengths_of_pieces(T, n):
    """In a table just long enough (tiles of short tables stay whole) and in a longer one."""
    for width in (None, -(-T // 16) + 1, 49, 300):
        if width is not None and width * 16 < T:
            continue
        Case([T, n], Hq=8, Hkv=2, D=64, length=[T], rows=[n], width=width).check()


@pytest.mark.parametrize("dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("prefix", [1, 900, 1027, 1500])
def test_tokens_with_tags_weigh_more_than_the_prefix(dtype, D, Hq, Hkv, prefix):
    c = Case([prefix, D], dtype, Hq, Hkv, D, 32, [1500, 700], [6, 64])
    c.check(see=c.rng.integers(-2 ** 63, 2 ** 63, c.n), prefix=[prefix, min(prefix, 700)])


@pytest.mark.parametrize("D,n", [(128, 3), (64, 9), (128, 35)])
def test_pieces_joined_from_few_parts_and_from_many(D, n):
    for T in (1100, 2300, 30000):
        Case([T, n], "f16", 4, 1, D, 64, [T], [n]).check()


@pytest.mark.parametrize("R", [15, 16, 17, 31, 32, 33, 63, 64, 65, 130])
def test_as_many_tiles_as_work_groups_that_run_at_once(R):
    rng = np.random.default_rng(R)
    length = rng.integers(1, 1400, R)
    Case([R, 2], "bf16", 8, 8, 64, length=length, rows=np.minimum(length, rng.integers(1, 3, R)), pad=3).check()


@pytest.mark.parametrize("seed", range(12))
def test_batches_of_any_kind(seed):
    """No part of a plan may go missing: what no work-group computes keeps its first value."""
    rng = np.random.default_rng([seed, 77])
    R = int(rng.integers(1, 12))
    Hkv = int(rng.choice([1, 2, 8]))
    G = int(rng.choice([1, 2, 4]))
    length = np.where(rng.random(R) < 0.2, 0, np.exp(rng.uniform(0, np.log(3000), R))).astype(int)
    rows = np.minimum(length, np.exp(rng.uniform(0, np.log(90), R)).astype(int))
    c = Case([seed, 5], ["bf16", "f16"][seed % 2], Hkv * G, Hkv, [64, 128][seed // 2 % 2], 16, length, rows, pad=int(rng.integers(0, 40)),
             width=None if seed % 3 else 400)
    tagged = rng.random() < 0.5
    c.check(see=rng.integers(-2 ** 63, 2 ** 63, c.n) if tagged else None, prefix=rng.integers(0, 1 + length) if rng.random() < 0.5 else None)


@pytest.mark.parametrize("dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [4, 40])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_positions_in_order_and_out_of_it(dtype, D, Hq, Hkv, n, cap):
    """A prompt's positions; then blocks that start anywhere, stand still, go down, or leave one gap; rows far behind, among and ahead of them."""
    c = Case([n, D], dtype, Hq, Hkv, D, 16, [900], [n])
    t = np.arange(900)
    pos = 40 + t
    for b in range(10, 56):
        at = slice(16 * b, min(16 * b + 16, 900))
        i = np.arange(at.stop - at.start)
        start = int(c.rng.integers(0, 1500))
        pos[at] = [start + i, start + 0 * i, start + 15 - i, start + i + (i > 9), start + i - (i == 15)][b % 5]
    c.position[c.table[0, t // 16] * 16 + t % 16] = pos
    row = c.rng.integers(30, 1500, n)
    row[0], row[1] = 2000, 40 + 15
    c.check(slopes=c.rng.uniform(-0.002, 0.02, Hq).astype(np.float32), row_position=row, cap=cap)
    c.check(slopes=np.full(Hq, 0.01, np.float32), row_position=np.full(n, 3000), cap=cap)


@pytest.mark.parametrize("R", [2, 3, 5, 16, 40, 100, 200])
@pytest.mark.parametrize("Hkv", [1, 8])
def test_requests_with_few_rows_beside_others_with_many(R, Hkv):
    """Their units weigh differently; none is lost whatever the weights make of the split."""
    rng = np.random.default_rng([R, Hkv, 50])
    length = rng.integers(1, 400 if R > 16 else 1500 if Hkv > 1 else 6000, R)
    rows = np.minimum(length, rng.integers(0, 9, R))
    rows[0], rows[1] = min(length[0], 1), min(length[1], 8)
    c = Case([R, Hkv, 51], "bf16", 4 * Hkv, Hkv, 64, 16, length, rows, width=400)
    c.check(prefix=np.where(rng.random(R) < 0.5, length // 2, 0))
    c.check(see=rng.integers(-2 ** 63, 2 ** 63, c.n), prefix=length // 3)
