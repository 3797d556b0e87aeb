"""Scores that fp32 no longer tells apart: the result is a mean of values of tokens whose scores are the row's largest within what fp32 holds of them, and finite.

What fp32 holds of a score: products of D terms, scale, distance and the differences to a base, each to 2^-24 of the row's largest magnitude; 2^-18 of it is more
than all of them together (128 terms' sums 2^-17 of a term's, of which the largest score has some hundred).  Thirty more take the weights of all others below 2^-40 of
the largest, 2^14 tokens together 2^-26.  A mean's weights enter as fp16, 2^-11 of each."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from test_gpu_kv4_attend import TD, Case

pytestmark = pytest.mark.gpu


def check(c, row_position=None, slopes=None, prefix=None):
    got, lse = c.run(row_position=row_position, slopes=slopes, prefix=None if prefix is None else [prefix] * c.R)
    assert np.isfinite(got).all() and np.isfinite(lse).all()
    k, v = c.c.natural()
    q, G = c.q.double().numpy(), c.Hq // c.Hkv
    eps = torch.finfo(TD[c.dtype]).eps
    for r in range(c.R):
        t = np.arange(int(c.length[r]))
        at = c.table[r, t // c.P] * c.P + t % c.P
        lo, n = c.offs[r], c.offs[r + 1] - c.offs[r]
        for i in range(n):
            p = int(c.length[r]) - n + i
            seen = (t <= p) | (t < (prefix or 0))
            for h in range(c.Hq):
                s = c.scale * (k[at, h // G] @ q[lo + i, h])
                if slopes is not None:
                    s = s - float(slopes[h]) * np.abs((int(row_position[lo + i]) - c.position[at]) if row_position is not None else p - t)
                s, x = s[seen], v[at, h // G][seen]
                large = np.abs(s).max()
                near = s >= s.max() - 2.0 ** -18 * large - 30.0
                off = (eps / 2 + 2.0 ** -10) * np.abs(x[near]).max(0) + 2.0 ** -20 * np.abs(x).max()
                o = got[lo + i, h]
                assert (o <= x[near].max(0) + off).all() and (o >= x[near].min(0) - off).all(), (r, i, h, float(s.max()))
                assert abs(lse[lo + i, h] - s.max()) <= 2.0 ** -18 * large + 30.0


@pytest.mark.parametrize("scale", [20, 24, 27, 30, -33, 50, 100])
@pytest.mark.parametrize("n", [1, 3, 7, 40])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 128), ("bf16", 64), ("f16", 64)])
def test_large_scales(dtype, D, n, scale):
    check(Case([n, abs(scale), D], dtype, 8, 2, D, 32, [300, 77], [n, 2], scale=float(np.copysign(2.0 ** abs(scale), scale))))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [2, 20])
@pytest.mark.parametrize("scale", [24, 30])
def test_large_scores_of_tokens_split_over_work_groups(scale, n, dtype):
    check(Case([n, scale, 5], dtype, 4, 1, 64, 32, [9000], [n], scale=2.0 ** scale))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [2, 40])
@pytest.mark.parametrize("first", ["small", "large"])
def test_large_scores_behind_small_ones_and_ahead(first, n, dtype):
    """Tokens whose K is 2^-40 of the others': scores near 0 and far from it, in either order."""
    c = Case([n, 6], dtype, 8, 2, 128, 16, [600], [n], scale=2.0 ** 30)
    t = np.arange(600)
    for i, s in enumerate(c.table[0, t // 16] * 16 + t % 16):
        if (i < 200) == (first == "small"):
            c.c.ks[s // 16, :, s % 16] -= 40
    check(c)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [2, 40])
@pytest.mark.parametrize("slope", [1.0, 2.0 ** 20, -3.0])
def test_rows_far_from_all_tokens(slope, n, dtype):
    """Scores of -2^30 and below, none of them near 0 (and, by a slope below zero, far above it)."""
    c = Case([n, 7], dtype, 8, 2, 64, 16, [300], [n])
    check(c, row_position=np.full(c.n, 2 ** 30), slopes=np.full(8, slope, np.float32))


@pytest.mark.parametrize("n", [2, 80])
def test_large_scores_under_a_prefix_in_batches(n):
    check(Case([n, 8], "bf16", 8, 2, 128, 16, [300, 90, 600], [n, 1, 5], scale=2.0 ** 28), prefix=280)
