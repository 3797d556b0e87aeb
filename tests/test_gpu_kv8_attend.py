"""Attention over the 8-bit cache against 64 bits, row by row and head by head.

Bound of an output's error, from what is rounded (w the softmax weights, which sum to 1, e = 2^-11 fp16's half step):
  the result to its type                  eps(out) / 2 * |out|
  each weight to fp16, and to at least    e * sum w |v|  +  T * 2^-25 * max |v|   (weights below fp16's smallest normal number)
  each score, in fp32: the product's 128 terms, scale, cap, distance: 2^-20 (1 + largest |score|, |cap|), twice in a weight's ratio
                                          2 * 2^-20 (1 + max |s| + cap) * sum w |v|
and of lse 2^-20 (1 + max |s| + cap + |lse|)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv8_ref as ref
from paper_2502_11517_amd import kv8

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f16": torch.float16}


def dev(a, dtype=torch.int32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


class Case:
    """Random codes and scales in scattered pages; everything that no request holds is poisoned (NaN codes, NaN scales)."""

    def __init__(self, seed, codes="e4m3", dtype="bf16", Hq=8, Hkv=2, D=128, P=16, length=(40,), rows=(3,), pad=0, scale=None, std=1.0, width=None,
                 spread=2):
        rng = self.rng = np.random.default_rng(seed)
        self.codes, self.dtype, self.Hq, self.Hkv, self.D, self.P = codes, dtype, Hq, Hkv, D, P
        self.length, self.R = np.asarray(length), len(length)
        self.offs = np.concatenate([[0], np.cumsum(rows)]).astype(int)
        self.n = int(self.offs[-1]) + pad
        need = [-(-int(x) // P) for x in length]
        self.W = width or max(1, max(need))
        self.pages = sum(need) + 2
        perm = rng.permutation(self.pages)
        self.table = np.full((self.R, self.W), -1)
        at = 0
        for r, k in enumerate(need):
            self.table[r, :k] = perm[at:at + k]
            at += k
        self.scale = D ** -0.5 if scale is None else scale
        B = P // 16
        val = ref.code_values(codes)
        top = 100 if codes == "e4m3" else 127
        shape = (self.pages, Hkv, B, 16, D)
        kb = rng.integers(0, top, shape).astype(np.uint8) | (rng.integers(0, 2, shape) << 7).astype(np.uint8)
        vb = rng.integers(0, top, shape).astype(np.uint8) | (rng.integers(0, 2, shape) << 7).astype(np.uint8)
        unit = 2.0 ** -4 if codes == "e4m3" else 2.0 ** -6
        ks = std * unit * 2.0 ** rng.integers(-spread, spread + 1, shape[:3])
        vs = unit * 2.0 ** rng.integers(-spread, spread + 1, shape[:3])
        held = np.zeros((self.pages, P), bool)
        for r in range(self.R):
            t = np.arange(int(length[r]))
            held[self.table[r, t // P], t % P] = True
        blocks = held.reshape(self.pages, B, 16).any(-1)
        bad = np.uint8(0x7f)
        kb[~blocks.repeat(Hkv, 0).reshape(self.pages, Hkv, B)] = bad
        vb[~blocks.repeat(Hkv, 0).reshape(self.pages, Hkv, B)] = bad
        ks[~blocks.repeat(Hkv, 0).reshape(self.pages, Hkv, B)] = np.nan
        vs[~blocks.repeat(Hkv, 0).reshape(self.pages, Hkv, B)] = np.nan
        self.kb, self.vb, self.ks, self.vs = kb, vb, ks, vs
        self.q = torch.from_numpy(rng.standard_normal((self.n, Hq, D)).astype(np.float32)).to(TD[dtype])
        self.tag = rng.integers(0, 64, self.pages * P)
        self.position = rng.integers(0, 5000, self.pages * P)
        self.val = val

    def natural(self):
        def one(b, s):
            with np.errstate(invalid="ignore"):
                x = self.val[b] * s[..., None, None]
            return x.transpose(0, 2, 3, 1, 4).reshape(self.pages * self.P, self.Hkv, self.D)
        return one(self.kb, self.ks), one(self.vb, self.vs)

    def config(self):
        return kv8.make_config(self.codes, self.dtype, self.Hq, self.Hkv, self.D, self.scale, max_requests=max(1, self.R), max_rows=max(1, self.n),
                               page_tokens=self.P, n_phys_pages=self.pages, pages_per_request=self.W)

    def run(self, *, prefix=None, cap=0.0, slopes=None, see=None, row_position=None, slot=None, most=None, stream=None):
        d = dict(k=dev(ref.k_stored(self.kb), torch.uint8), v=dev(np.moveaxis(self.vb, -1, -2), torch.uint8), ks=dev(self.ks, torch.float32),
                 vs=dev(self.vs, torch.float32), table=dev(self.table), tag=dev(self.tag, torch.uint8), position=dev(self.position))
        cfg = self.config()
        q = self.q.cuda()
        out, lse = torch.full_like(q, 7.0), torch.full((self.n, self.Hq), 7.0, device="cuda")
        ws = torch.full((kv8.query_workspace_bytes(cfg),), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        s = stream or torch.cuda.current_stream()
        h = kv8.PastaKv8(cfg, ws, page_table=d["table"], k_codes=d["k"], v_codes=d["v"], k_scale=d["ks"], v_scale=d["vs"], slot_tag=d["tag"],
                         slot_position=d["position"], stream=s.cuda_stream)
        h.plan(dev(self.length), dev(self.offs), self.n, max_request_rows=most, prefix_len=dev(prefix), slot=dev(slot))
        h.attend(0, q, out, lse=lse, logit_cap=cap, slopes=dev(slopes, torch.float32), row_see=dev(see, torch.int64), row_position=dev(row_position))
        torch.cuda.synchronize()
        return out.double().cpu().numpy(), lse.double().cpu().numpy()

    def check(self, *, refused=(), rel_s=1.0, **kw):
        got, lse = self.run(**kw)
        kw.pop("most", None), kw.pop("slot", None), kw.pop("stream", None)
        k, v = self.natural()
        cap, see = kw.get("cap", 0.0), kw.pop("see", None)
        want, wlse, mean, most_v, most_s = ref.attend(self.q.double().numpy(), k, v, self.length, self.offs, self.table, self.P, scale=self.scale,
                                                      G=self.Hq // self.Hkv, tag=self.tag, see=see, position=self.position, refused=refused, **kw)
        T = max([1, *self.length])
        ds = 2.0 ** -20 * (1 + most_s + cap)
        eps = torch.finfo(TD[self.dtype]).eps
        bound = eps / 2 * np.abs(want) + (2.0 ** -11 + 2 * ds[..., None]) * mean + T * 2.0 ** -25 * most_v[..., None] + 1e-30
        bound *= 1 + 2.0 ** -6  # (second order)
        nan = np.isnan(wlse)
        assert np.array_equal(np.isnan(lse), nan) and np.isnan(got[nan]).all()
        off = np.abs(got - want)[~nan]
        assert (off <= bound[~nan]).all(), float((off / bound[~nan]).max())
        fin = np.isfinite(wlse)
        assert np.array_equal(np.isneginf(lse), np.isneginf(wlse))
        off = np.abs(lse - wlse)[fin] / (2.0 ** -20 * (1 + most_s + cap + np.abs(wlse)))[fin]
        assert (off <= 1).all(), float(off.max())
        return got, lse


SHAPES = [("e4m3", "bf16", 128, 8, 2), ("int8", "f16", 64, 4, 4), ("e4m3", "f16", 64, 16, 2), ("int8", "bf16", 128, 4, 2)]


@pytest.mark.parametrize("codes,dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 500, 2049])
def test_one_row_over_lengths_of_every_kind(codes, dtype, D, Hq, Hkv, P, T):
    Case([T, P], codes, dtype, Hq, Hkv, D, P, [T], [1]).check()


@pytest.mark.parametrize("codes,dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n,T", [(2, 2), (7, 40), (8, 300), (9, 77), (31, 31), (33, 200), (65, 130), (100, 1000), (150, 333)])
def test_pieces_of_prompts(codes, dtype, D, Hq, Hkv, n, T):
    Case([n, T], codes, dtype, Hq, Hkv, D, 32, [T], [n]).check()


@pytest.mark.parametrize("wide", [False, True])
def test_batches_of_ragged_requests(wide):
    length = [0, 5, 700, 33, 1, 260, 64, 0, 129, 1500]
    rows = [0, 2, 1, 8, 1, 40 if wide else 3, 0, 0, 64 if wide else 7, 4]
    Case(5, length=length, rows=rows, pad=9).check()


def test_more_requests_than_a_wave_has_lanes():
    rng = np.random.default_rng(6)
    length = rng.integers(1, 90, 300)
    Case(6, "int8", "f16", 4, 4, 64, length=length, rows=np.minimum(length, rng.integers(0, 3, 300))).check()


@pytest.mark.parametrize("T,n", [(20000, 2), (9000, 40)])
def test_tokens_split_over_many_work_groups(T, n):
    Case([T, n], Hq=4, Hkv=1, D=64, P=16, length=[T], rows=[n]).check()


def test_rows_beyond_the_stated_most_are_still_right():
    Case(8, length=[300, 40], rows=[60, 3]).check(most=1)
    Case(8, length=[300, 40], rows=[5, 3]).check(most=8)


@pytest.mark.parametrize("scale", [0.0, -0.11, 0.7])
@pytest.mark.parametrize("n", [3, 40])
def test_scales_of_every_sign(scale, n):
    Case([n, 9], length=[150], rows=[n], scale=scale).check()


@pytest.mark.parametrize("codes,dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("cap", [5.0, 50.0])
def test_capped_scores(codes, dtype, D, Hq, Hkv, n, cap):
    Case([n, int(cap)], codes, dtype, Hq, Hkv, D, 16, [200, 60], [n, 3], std=3.0).check(cap=cap)


@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("given", [False, True])
def test_scores_lowered_by_distance(n, given):
    c = Case([n, given], "int8", "f16", 8, 2, 64, 32, [300, 77], [n, 5])
    slopes = c.rng.uniform(-0.01, 0.5, 8).astype(np.float32) * (0.02 if given else 1.0)
    c.check(slopes=slopes, row_position=c.rng.integers(0, 5000, c.n) if given else None, cap=20.0 if given else 0.0)


@pytest.mark.parametrize("n", [4, 50])
def test_tags_and_a_prefix(n):
    c = Case([n, 3], length=[300, 77, 64], rows=[n, 6, 2])
    see = c.rng.integers(-2 ** 63, 2 ** 63, c.n)
    see[1], see[n], see[n + 1] = 0, 0, 1 << 62
    c.check(see=see)
    c.check(see=see, prefix=[100, 0, 500])
    c.check(prefix=[295, 77, 1], see=np.zeros(c.n, np.int64))
    c.check(prefix=[290, 75, 0])  # tokens ahead of the row are seen within the prefix


@pytest.mark.parametrize("n", [4, 50])
def test_rows_that_see_nothing(n):
    c = Case([n, 4], length=[200], rows=[n])
    c.tag[:] = 5
    out, lse = c.check(see=np.where(np.arange(n) % 2, 1 << 5, ~(1 << 5)))
    assert (out[0::2] == 0).all() and np.isneginf(lse[0::2]).all() and np.isfinite(lse[1::2]).all()


@pytest.mark.parametrize("codes,dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [5, 70, 161])
@pytest.mark.parametrize("tags,cap", [(True, 0.0), (True, 20.0), (False, 20.0)])
def test_everything_at_once_over_split_tokens(codes, dtype, D, Hq, Hkv, n, tags, cap):
    c = Case([n, tags, int(cap)], codes, dtype, Hq, Hkv, D, 16, [1700, 0, 230], [n, 0, 3])
    see = c.rng.integers(-2 ** 63, 2 ** 63, c.n)
    see[n // 2] = 0
    slopes = c.rng.uniform(0.0, 0.01, Hq).astype(np.float32)
    c.check(see=see if tags else None, prefix=[90, 0, 17], cap=cap, slopes=slopes, row_position=c.rng.integers(0, 1700, c.n) if tags else None)


def test_streams_with_blocks_of_one_tag_and_of_many():
    c = Case(11, length=[260], rows=[8])
    for r in range(1):
        t = np.arange(260)
        c.tag[c.table[r, t // c.P] * c.P + t % c.P] = np.where(t < 100, 1, np.where(t < 150, 2 + t % 8, 2 + t // 16 % 8))
    c.check(see=np.array([(1 << 1) | (1 << (2 + i)) for i in range(8)]))


@pytest.mark.parametrize("n", [4, 50])
def test_nan_blocks_reach_only_rows_that_see_them(n):
    for which in ("ks", "vs", "both"):
        c = Case([n, 12], length=[200], rows=[n])
        c.tag[:] = 0
        page = c.table[0, 3]
        c.tag[page * 16:page * 16 + 16] = 9
        if which != "vs":
            c.ks[page] = np.nan
        if which != "ks":
            c.vs[page, 1] = np.nan
        see = np.where(np.arange(n) % 2, 1, 1 | 1 << 9)
        out, lse = c.run(see=see)
        k, v = c.natural()
        want = ref.attend(c.q.double().numpy(), k, v, c.length, c.offs, c.table, 16, scale=c.scale, G=4, tag=c.tag, see=see)
        assert np.array_equal(np.isnan(out), np.isnan(want[0])) and np.array_equal(np.isnan(lse), np.isnan(want[1]))
        assert np.isnan(out[0]).any() and not np.isnan(out[1::2]).any()
        fin = ~np.isnan(want[0])
        assert np.abs(out - want[0])[fin].max() < 0.02 * np.abs(want[0])[fin].max()


def test_rows_of_infinite_and_nan_queries_stay_alone():
    c = Case(13, length=[90], rows=[5])
    c.q[1, 2, 7], c.q[3, 5, 0], c.q[0, 0, 0] = float("inf"), float("nan"), 3e38
    out, lse = c.run()
    good = np.ones((5, 8), bool)
    good[1, 2] = good[3, 5] = good[0, 0] = False
    assert np.isnan(out[1, 2]).all() and np.isnan(out[3, 5]).all() and np.isfinite(out[good]).all()
    k, v = c.natural()
    want = ref.attend(c.q.double().numpy(), k, v, c.length, c.offs, c.table, 16, scale=c.scale, G=4)[0]
    assert np.abs(out - want)[good].max() < 0.02 * np.abs(want[good]).max()


@pytest.mark.parametrize("size", [1e-30, 1e-4, 1e4])
def test_queries_of_every_size(size):
    c = Case(14, "e4m3", "bf16", length=[100], rows=[3], scale=1.0 / size / 12)
    c.q = (c.q.float() * size).to(torch.bfloat16)
    c.check()


def test_scores_far_apart():
    Case(15, length=[400], rows=[3], std=40.0).check()
    Case(15, length=[400], rows=[40], std=40.0).check()


@pytest.mark.parametrize("n", [3, 40])
def test_scales_of_v_far_apart(n):
    """Weights lose nothing of fp16's 11 bits for blocks 2^13 below the largest: 2^-14 of it is fp16's smallest normal number."""
    c = Case([n, 16], length=[300], rows=[n], spread=6)
    c.check()
    c.vs[:] = np.where(np.isnan(c.vs), np.nan, 2.0 ** -100)
    c.check()
    c.vs[c.table[0, 5]] = 2.0 ** 100
    got, _ = c.run()
    assert np.isfinite(got).all() == (c.dtype != "f16")


@pytest.mark.parametrize("n", [3, 40])
def test_pages_with_bad_numbers_are_seen_by_nobody(n):
    c = Case([n, 17], length=[200, 40], rows=[n, 4])
    c.table[0, 2], c.table[0, 3], c.table[0, 9], c.table[1, 2] = -1, 1 << 29, c.pages, -(1 << 31)
    c.check()
    c.table[1, :] = -1
    out, lse = c.check(see=np.full(c.n, -1))
    assert (out[n:] == 0).all() and np.isneginf(lse[n:]).all()


def test_refused_requests_and_padding_get_rows_that_see_nothing():
    c = Case(18, length=[100, 50, 30], rows=[2, 40, 3], pad=70)
    slot = np.zeros(c.n, int)
    slot[2:42] = -1
    out, lse = c.check(slot=slot, refused=(1,))
    assert (out[2:42] == 0).all() and np.isneginf(lse[2:42]).all() and (out[45:] == 0).all() and np.isneginf(lse[45:]).all()


def test_lengths_and_offsets_that_are_wrong_stay_inside_the_arrays():
    c = Case(19, length=[100, 50], rows=[2, 3], width=7)
    c.length = np.array([1 << 30, -9])
    c.run()
    c.offs = np.array([0, 1 << 20, 3])
    c.run()
    c.offs = np.array([-5, 4, 2])
    c.run()


def test_work_on_another_stream():
    s = torch.cuda.Stream()
    Case(20, length=[500], rows=[8]).check(stream=s)


def test_layers_beyond_four_gibibytes():
    H, D, P = 8, 128, 64
    pages = (5 << 30) // (H * D * P)
    c = Case(21, Hq=16, Hkv=H, D=D, P=P, length=[100], rows=[4])
    want, wlse = c.run()
    cfg = kv8.make_config("e4m3", "bf16", 16, H, D, c.scale, max_rows=4, page_tokens=P, n_phys_pages=pages, pages_per_request=2)
    k = torch.zeros(kv8.cache_shapes(cfg)[0], dtype=torch.uint8, device="cuda")
    v = torch.zeros(kv8.cache_shapes(cfg)[1], dtype=torch.uint8, device="cuda")
    ks, vs = torch.zeros(kv8.cache_shapes(cfg)[2], device="cuda"), torch.zeros(kv8.cache_shapes(cfg)[2], device="cuda")
    table = [pages - 1, pages // 2]
    for at, page in zip(table, c.table[0]):
        k[0, at], v[0, at] = dev(ref.k_stored(c.kb)[page], torch.uint8), dev(np.moveaxis(c.vb[page], -1, -2), torch.uint8)
        ks[0, at], vs[0, at] = dev(c.ks[page], torch.float32), dev(c.vs[page], torch.float32)
    q = c.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(4, 16, device="cuda")
    h = kv8.PastaKv8(cfg, torch.empty(kv8.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), page_table=dev([table]), k_codes=k, v_codes=v,
                     k_scale=ks, v_scale=vs, stream=torch.cuda.current_stream().cuda_stream)
    h.plan(dev([100]), dev([0, 4]), 4)
    h.attend(0, q, out, lse=lse)
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want) and np.array_equal(lse.double().cpu().numpy(), wlse)
