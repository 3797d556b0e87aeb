"""Caps of every size.  A cap far above the scores leaves them as they are, however high it is; one far below brings them all to it.

Bounds are those of test_gpu_kv8_attend but for the cap's own part of a score's error.  The closed form of cap * tanh(x / cap) rounds a few numbers of the
cap's size: 2^-20 cap covers them.  It is taken for caps up to 128 / log2(e) = 88, and else only for |x| > cap / 8: 2^-20 * min(cap, 8 max |x|)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv8_ref as ref
from test_gpu_kv8_attend import SHAPES, TD, Case, pytestmark  # noqa: F401


def check(c, cap, see=None, slopes=None):
    got, lse = c.run(cap=cap, see=see, slopes=slopes)
    k, v = c.natural()
    cap = float(np.float32(cap))
    args = (c.q.double().numpy(), k, v, c.length, c.offs, c.table, c.P)
    kw = dict(scale=c.scale, G=c.Hq // c.Hkv, tag=c.tag, see=see, slopes=slopes)
    want, wlse, mean, most_v, most_s = ref.attend(*args, cap=cap, **kw)
    most_x = ref.attend(*args, **{**kw, "slopes": None})[4]
    assert np.isfinite(wlse).all()
    ds = 2.0 ** -20 * (1 + most_s + (cap if cap <= 88 else np.minimum(cap, 8 * most_x)))
    bound = torch.finfo(TD[c.dtype]).eps / 2 * np.abs(want) + (2.0 ** -11 + 2 * ds[..., None]) * mean + max(c.length) * 2.0 ** -25 * most_v[..., None]
    off = np.abs(got - want)
    assert (off <= bound * (1 + 2.0 ** -6)).all(), float((off / bound).max())
    assert (np.abs(lse - wlse) <= ds + 2.0 ** -20 * np.abs(wlse)).all(), float((np.abs(lse - wlse) / (ds + 2.0 ** -20 * np.abs(wlse))).max())


@pytest.mark.parametrize("codes,dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("cap", [88.0, 90.0, 300.0, 1e4, 1e9, 1e30, 3.4e38])
def test_high_caps(codes, dtype, D, Hq, Hkv, n, cap):
    """Scores around 1, and of 40 to 100 so that some are past an eighth of the lower caps."""
    for std in (1.0, 40.0):
        check(Case([n, D], codes, dtype, Hq, Hkv, D, 16, [200, 60], [n, 3], std=std), cap)


@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("cap", [1e-3, 1e-20, 1e-30, 1e-39, 1e-45])
def test_low_caps(n, cap):
    check(Case([n, 1], length=[200, 60], rows=[n, 3]), cap)


@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("cap", [50.0, 1e6])
def test_high_caps_with_tags_and_distances(n, cap):
    c = Case([n, 2], "int8", "f16", 8, 2, 64, 32, [300, 77], [n, 5])
    check(c, cap, see=c.rng.integers(0, 2 ** 62, c.n) | 1, slopes=c.rng.uniform(0.0, 0.01, 8).astype(np.float32))
