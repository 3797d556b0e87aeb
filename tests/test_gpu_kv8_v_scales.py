"""Attention over blocks whose V scales lie up to 2^200 apart, against 64 bits: sums and lse know nothing of V's scales, wherever the blocks lie and
whichever wave, stretch of blocks or part of the tokens they come to.

Bounds, with w the softmax weights, u = w * (V's scale) and M the row's largest u:
  out   half a step of its type, 2^-11 of each weight (fp16), and 2^-25 M of weights that are small in units of M, but no more than those:
        eps / 2 |out| + (2^-11 + 2 ds) sum w |v| + sum min(u, 2^-25 M) |code|
  lse   2^-20 (1 + max |s| + |lse|) as in test_gpu_kv8_attend, and the roundings of numbers as large as the scales' exponents (at most 128, in log2 units):
        of the base, of what is subtracted from it, of log2 of the sum (two halves of a step) -- 4 * 2^-24 * 128 * ln 2;  ds is the same without |lse|"""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_kv8_attend import TD, Case, pytestmark  # noqa: F401
import torch

APART = 4 * 2.0 ** -24 * 128 * np.log(2)


def check(c, see=None):
    """One request; every row and head from the definition."""
    got, got_lse = c.run(see=see)
    T, n, G = int(c.length[0]), c.n, c.Hq // c.Hkv
    t = np.arange(T)
    page, block, in_block = c.table[0, t // c.P], t % c.P // 16, t % 16
    eps, q = torch.finfo(TD[c.dtype]).eps, c.q.double().numpy()
    for i in range(n):
        vis = t <= T - n + i
        if see is not None:
            vis &= np.array([(int(see[i]) >> int(g)) & 1 for g in c.tag[page * c.P + t % c.P]], bool)
        assert vis.any()
        for h in range(c.Hq):
            at = (page[vis], h // G, block[vis])
            s = (c.val[c.kb[at + (in_block[vis],)]] * c.ks[at][:, None]) @ q[i, h] * c.scale
            code, vs = c.val[c.vb[at + (in_block[vis],)]], c.vs[at]
            m = s.max()
            w = np.exp(s - m)
            lse = m + np.log(w.sum())
            w /= w.sum()
            u = w * vs
            want = u @ code
            ds = 2.0 ** -20 * (1 + np.abs(s).max()) + APART
            bound = eps / 2 * np.abs(want) + (2.0 ** -11 + 2 * ds) * (u @ np.abs(code)) + np.minimum(u, 2.0 ** -25 * u.max()) @ np.abs(code)
            off = np.abs(got[i, h] - want)
            assert (off <= bound * (1 + 2.0 ** -6)).all(), (i, h, float((off / bound).max()))
            assert abs(got_lse[i, h] - lse) <= 2.0 ** -20 * (1 + np.abs(s).max() + abs(lse)) + APART, (i, h, got_lse[i, h], lse)


def case(seed, T, n, *, hkv=2, d=64, codes="e4m3", wide_table=True, **kw):
    return Case([seed, T, n], codes, "bf16", 4 * hkv, hkv, d, 16, [T], [n], width=300 if wide_table and T < 4800 else None, spread=0, **kw)


def pages(c, blocks):
    return c.table[0, np.asarray(blocks)]


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("wide_table", [False, True])
@pytest.mark.parametrize("big", [0, 5, 12, 18])
def test_one_block_far_above_the_others(n, wide_table, big):
    """Among the blocks of another wave and of its own; a short table is not split, a long one is."""
    for high, low in ((100, -100), (63, -63), (65, -65), (119, 0)):
        c = case(big, 300, n, wide_table=wide_table)
        c.vs[pages(c, range(19))] = 2.0 ** low
        c.vs[pages(c, [big])] = 2.0 ** high
        check(c)


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("big", [[0], [311], [70, 71], [130, 250], list(range(40, 80))])
def test_over_many_parts_and_stretches_of_blocks(n, big):
    c = case(1, 5000, n, hkv=1)
    c.vs[pages(c, range(313))] = 2.0 ** -100
    c.vs[pages(c, big)] = 2.0 ** 100
    check(c)


@pytest.mark.parametrize("hkv", [2, 8])
@pytest.mark.parametrize("first", [True, False])
def test_within_one_unit_longer_than_a_stretch(hkv, first):
    """Enough requests' worth of heads that a work-group reads more blocks than it lists; the large ones come early or late."""
    c = case(2, 4000, 40, hkv=hkv, d=128)
    c.vs[pages(c, range(250))] = 2.0 ** -100
    c.vs[pages(c, range(3) if first else range(247, 250))] = 2.0 ** 90
    check(c)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("T", [120, 700, 2500])
def test_scales_of_every_size_at_once(codes, n, T):
    c = case(3, T, n, codes=codes)
    held = ~np.isnan(c.vs)
    c.vs[held] = 2.0 ** c.rng.choice([-100, -90, -40, 0, 20, 59, 61, 100], int(held.sum()))
    check(c)


@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("T", [200, 2500])
def test_a_block_that_a_row_does_not_see_leaves_its_result_alone(n, T):
    """Odd rows see only blocks of 2^-100 beside one of 2^100 that is hidden from them."""
    c = case(4, T, n)
    c.tag[:] = 0
    c.vs[pages(c, range(-(-T // 16)))] = 2.0 ** -100
    hidden = pages(c, [6])
    c.vs[hidden] = 2.0 ** 100
    c.tag[hidden[0] * 16:hidden[0] * 16 + 16] = 9
    check(c, see=np.where(np.arange(n) % 2, 1, 1 | 1 << 9))
