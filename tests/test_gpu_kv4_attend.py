"""Attention over the 4-bit cache against 64 bits, row by row and head by head.

Bound of an output's error, from what is rounded (w the softmax weights, which sum to 1, e = 2^-11 fp16's half step):
  the result to its type                  eps(out) / 2 * |out|
  each weight to fp16                     e * sum w |v|  +  T * 2^-25 * max |v|   (weights below fp16's smallest normal number: half a step of 2^-24, in units of
                                          which the largest has 2^-1 at least: it is lifted by 2^7 and lowered by its V scale's distance from the block's, 2^-8)
  each score, in fp32: the product's 128 terms (twice as many in two parts), scale, cap, distance: 2^-20 (1 + largest |score|, |cap|), twice in a weight's ratio
                                          2 * 2^-20 (1 + max |s| + cap) * sum w |v|
and of lse 2^-20 (1 + max |s| + cap + |lse|)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2502_11517_amd import kv4

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f16": torch.float16}


def dev(a, dtype=torch.int32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


class Case:
    """Random codes and scales in scattered pages; everything that no request holds has scales that are not numbers."""

    def __init__(self, seed, dtype="bf16", Hq=8, Hkv=2, D=128, P=16, length=(40,), rows=(3,), pad=0, scale=None, std=1.0, width=None, spread=2, k_spread=2):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.Hq, self.Hkv, self.D, self.P = dtype, Hq, Hkv, D, P
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
        shape = (self.pages, Hkv, P)
        unit = 127 - 1 + int(round(np.log2(std)))
        self.c = ref.Cache(self.pages, Hkv, P, D, rng.integers(0, 16, (*shape, D)).astype(np.uint8), rng.integers(0, 16, (*shape, D)).astype(np.uint8),
                           (unit + rng.integers(-k_spread, k_spread + 1, (*shape, D // 32))).astype(np.uint8),
                           (126 + rng.integers(-spread, spread + 1, shape)).astype(np.uint8))
        held = np.zeros((self.pages, P), bool)
        for r in range(self.R):
            t = np.arange(int(length[r]))
            held[self.table[r, t // P], t % P] = True
        self.c.ks[~np.broadcast_to(held[:, None, :], shape)] = ref.NONE
        self.c.vs[~np.broadcast_to(held[:, None, :], shape)] = ref.NONE
        self.q = torch.from_numpy(rng.standard_normal((self.n, Hq, D)).astype(np.float32)).to(TD[dtype])
        self.tag = rng.integers(0, 64, self.pages * P)
        self.position = rng.integers(0, 5000, self.pages * P)

    def config(self):
        return kv4.make_config(self.dtype, self.Hq, self.Hkv, self.D, self.scale, max_requests=max(1, self.R), max_rows=max(1, self.n), page_tokens=self.P,
                               n_phys_pages=self.pages, pages_per_request=self.W)

    def run(self, *, prefix=None, cap=0.0, slopes=None, see=None, row_position=None, slot=None, most=None, stream=None):
        cfg = self.config()
        bufs = [dev(b, torch.uint8).reshape(s) for b, s in zip(self.c.pack(), kv4.cache_shapes(cfg))]
        table, tag, position = dev(self.table), dev(self.tag, torch.uint8), dev(self.position)
        q = self.q.cuda()
        out, lse = torch.full_like(q, 7.0), torch.full((self.n, self.Hq), 7.0, device="cuda")
        ws = torch.full((kv4.query_workspace_bytes(cfg),), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        s = stream or torch.cuda.current_stream()
        h = kv4.PastaKv4(cfg, ws, page_table=table, k_codes=bufs[0], v_codes=bufs[1], k_scale=bufs[2], v_scale=bufs[3], slot_tag=tag, slot_position=position,
                         stream=s.cuda_stream)
        h.plan(dev(self.length), dev(self.offs), self.n, max_request_rows=most, prefix_len=dev(prefix), slot=dev(slot))
        h.attend(0, q, out, lse=lse, logit_cap=cap, slopes=dev(slopes, torch.float32), row_see=dev(see, torch.int64), row_position=dev(row_position))
        torch.cuda.synchronize()
        return out.double().cpu().numpy(), lse.double().cpu().numpy()

    def want(self, see=None, **kw):
        k, v = self.c.natural()
        return ref.attend(self.q.double().numpy(), k, v, self.length, self.offs, self.table, self.P, scale=self.scale, G=self.Hq // self.Hkv, tag=self.tag,
                          see=see, position=self.position, **kw)

    def check(self, *, refused=(), **kw):
        got, lse = self.run(**kw)
        kw.pop("most", None), kw.pop("slot", None), kw.pop("stream", None)
        want, wlse, mean, most_v, most_s = self.want(refused=refused, **kw)
        cap, T = kw.get("cap", 0.0), max([1, *self.length])
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
        off = np.abs(lse[fin] - wlse[fin]) / (2.0 ** -20 * (1 + most_s[fin] + cap + np.abs(wlse[fin])))
        assert (off <= 1).all(), float(off.max())
        return got, lse


SHAPES = [("bf16", 128, 8, 2), ("f16", 64, 4, 4), ("f16", 128, 16, 2), ("bf16", 64, 4, 2)]


@pytest.mark.parametrize("dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 500, 2049])
def test_one_row_over_lengths_of_every_kind(dtype, D, Hq, Hkv, P, T):
    Case([T, P], dtype, Hq, Hkv, D, P, [T], [1]).check()


@pytest.mark.parametrize("dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n,T", [(2, 2), (7, 40), (8, 300), (9, 77), (31, 31), (33, 200), (65, 130), (100, 1000), (150, 333)])
def test_pieces_of_prompts(dtype, D, Hq, Hkv, n, T):
    Case([n, T], dtype, Hq, Hkv, D, 32, [T], [n]).check()


@pytest.mark.parametrize("wide", [False, True])
def test_batches_of_ragged_requests(wide):
    length = [0, 5, 700, 33, 1, 260, 64, 0, 129, 1500]
    rows = [0, 2, 1, 8, 1, 40 if wide else 3, 0, 0, 64 if wide else 7, 4]
    Case(5, length=length, rows=rows, pad=9).check()


def test_more_requests_than_a_wave_has_lanes():
    rng = np.random.default_rng(6)
    length = rng.integers(1, 90, 300)
    Case(6, "f16", 4, 4, 64, length=length, rows=np.minimum(length, rng.integers(0, 3, 300))).check()


@pytest.mark.parametrize("T,n", [(20000, 2), (9000, 40)])
def test_tokens_split_over_many_work_groups(T, n):
    Case([T, n], Hq=4, Hkv=1, D=64, P=16, length=[T], rows=[n]).check()


def test_rows_beyond_the_stated_most_are_still_right():
    Case(8, length=[300, 40], rows=[60, 3]).check(most=1)
    Case(8, length=[300, 40], rows=[5, 3]).check(most=8)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [0.0, -0.11, 0.7])
@pytest.mark.parametrize("n", [3, 40])
def test_scales_of_every_sign(dtype, scale, n):
    Case([n, 9], dtype, length=[150], rows=[n], scale=scale).check()


@pytest.mark.parametrize("dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("cap", [5.0, 50.0])
def test_capped_scores(dtype, D, Hq, Hkv, n, cap):
    Case([n, int(cap)], dtype, Hq, Hkv, D, 16, [200, 60], [n, 3], std=4.0).check(cap=cap)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [4, 50])
@pytest.mark.parametrize("given", [False, True])
def test_scores_lowered_by_distance(dtype, n, given):
    c = Case([n, given], dtype, 8, 2, 64, 32, [300, 77], [n, 5])
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


@pytest.mark.parametrize("dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [5, 70, 161])
@pytest.mark.parametrize("tags,cap", [(True, 0.0), (True, 20.0), (False, 20.0)])
def test_everything_at_once_over_split_tokens(dtype, D, Hq, Hkv, n, tags, cap):
    c = Case([n, tags, int(cap)], dtype, Hq, Hkv, D, 16, [1700, 0, 230], [n, 0, 3])
    see = c.rng.integers(-2 ** 63, 2 ** 63, c.n)
    see[n // 2] = 0
    slopes = c.rng.uniform(0.0, 0.01, Hq).astype(np.float32)
    c.check(see=see if tags else None, prefix=[90, 0, 17], cap=cap, slopes=slopes, row_position=c.rng.integers(0, 1700, c.n) if tags else None)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_heads_that_share_a_kv_head(G):
    Case([G, 10], "bf16", 3 * G, 3, 128, 16, [150], [37]).check()


def test_streams_with_blocks_of_one_tag_and_of_many():
    c = Case(11, length=[260], rows=[8])
    t = np.arange(260)
    c.tag[c.table[0, t // c.P] * c.P + t % c.P] = np.where(t < 100, 1, np.where(t < 150, 2 + t % 8, 2 + t // 16 % 8))
    c.check(see=np.array([(1 << 1) | (1 << (2 + i)) for i in range(8)]))


@pytest.mark.parametrize("dtype,D,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("n", [4, 80])
def test_tokens_that_are_not_numbers_reach_only_rows_that_see_them(dtype, D, Hq, Hkv, n):
    for which in ("k", "v", "both"):
        c = Case([n, 12], dtype, Hq, Hkv, D, length=[200], rows=[n])
        c.tag[:] = 0
        slots = [c.table[0, t // 16] * 16 + t % 16 for t in (3, 49, 50, 66)]
        c.tag[slots] = 9
        for s in slots:
            if which != "v":
                c.c.ks[s // 16, 0, s % 16, (s * 7) % (D // 32)] = ref.NONE
            if which != "k":
                c.c.vs[s // 16, Hkv - 1, s % 16] = ref.NONE
        see = np.where(np.arange(n) % 2, 1, 1 | 1 << 9)
        out, lse = c.run(see=see)
        want = c.want(see=see)
        assert np.array_equal(np.isnan(lse), np.isnan(want[1])) and np.array_equal(np.isnan(out), np.isnan(want[0]))
        assert np.isnan(out[0]).any() and not np.isnan(out[1::2]).any()
        fin = ~np.isnan(want[0])
        assert np.abs(out - want[0])[fin].max() < 0.02 * np.abs(want[0])[fin].max()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_of_infinite_and_nan_queries_stay_alone(dtype):
    c = Case(13, dtype, length=[90], rows=[5])
    c.q[1, 2, 7], c.q[3, 5, 0] = float("inf"), float("nan")
    out, lse = c.run()
    good = np.ones((5, 8), bool)
    good[1, 2] = good[3, 5] = False
    assert np.isnan(out[1, 2]).all() and np.isnan(out[3, 5]).all() and np.isfinite(out[good]).all()
    want = c.want()[0]
    assert np.abs(out - want)[good].max() < 0.02 * np.abs(want[good]).max()


@pytest.mark.parametrize("dtype,size", [("bf16", 1e-30), ("bf16", 1e-4), ("bf16", 1e4), ("bf16", 1e30), ("f16", 1e-3), ("f16", 1e4)])
def test_queries_of_every_size(dtype, size):
    c = Case(14, dtype, length=[100], rows=[3], scale=1.0 / size / 12)
    c.q = (c.q.float() * size).to(TD[dtype])
    c.check()


def test_small_numbers_of_fp16_are_kept():
    c = Case(24, "f16", length=[100], rows=[3], scale=2.0 ** 17)
    c.q = (c.q.float() * 2.0 ** -20).to(torch.float16)
    assert (c.q.abs() < 2.0 ** -14).all()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scores_far_apart(dtype):
    Case(15, dtype, length=[400], rows=[3], std=32.0).check()
    Case(15, dtype, length=[400], rows=[40], std=32.0).check()


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("spread", [0, 1, 4, 5, 6, 20, 45])
def test_scales_of_v_far_apart(n, spread):
    """Within a block and between blocks: both sides of what a block's weights bear."""
    for dtype in ("bf16", "f16") if spread < 12 else ("bf16",):  # (fp16 ends at 2^16)
        Case([n, 16, spread], dtype, length=[300], rows=[n], spread=spread).check()


@pytest.mark.parametrize("n", [3, 40])
def test_scales_of_v_at_the_ends_of_their_range(n):
    c = Case([n, 26], length=[300], rows=[n])
    held = c.c.vs != ref.NONE
    for byte in (27, 246):
        c.c.vs[held] = byte
        if byte == 27:
            c.check()
        out, _ = c.run()
        assert np.isfinite(out).all()
    c.c.vs[held] = 27
    s = c.table[0, 3] * 16 + 5  # one token whose V is 2^200 times the others'
    c.c.vs[s // 16, :, s % 16] = 227
    c.check()


@pytest.mark.parametrize("n", [3, 40])
def test_rows_of_v_that_are_zero(n):
    """A V row of zeros lies under the least scale; it counts in the sums."""
    c = Case([n, 27], length=[300], rows=[n])
    for t in (0, 1, 17, 40, 41, 250, *range(64, 96)):
        s = c.table[0, t // 16] * 16 + t % 16
        c.c.vc[s // 16, :, s % 16], c.c.vs[s // 16, :, s % 16] = 0, 27
    c.check()


@pytest.mark.parametrize("n", [3, 40])
def test_scales_of_k_far_apart(n):
    c = Case([n, 28], length=[300], rows=[n], k_spread=6)
    c.check()
    c.c.ks[c.c.ks != ref.NONE] = 27
    c.check()


@pytest.mark.parametrize("n", [8, 80])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("far", [10, 12, 13, 14, 18, 24, 30, 34])
@pytest.mark.parametrize("down", [False, True])
def test_scales_of_k_beyond_a_window_of_fp16(n, D, far, down):
    """Groups of dims 2^far apart, in all tokens, in some, and not a number in one; rows that see one group, the other, or both, in sizes that make scores of 1.
    (Where only some tokens have the small scale, the rows made for it see those alone: the others' scores would be 2^far, and from 2^22 on fp32 does not tell
    scores apart.)"""
    for some in (False, True):
        c = Case([n, D, far, down, some], "f16", 8, 2, D, length=[300], rows=[n], scale=2.0 ** 14, k_spread=0)
        t = np.arange(300)
        slots = c.table[0, t // 16] * 16 + t % 16
        c.tag[:] = 2
        for i, s in enumerate(slots):
            k = c.c.ks[s // 16, :, s % 16]
            k[:] = 127
            if not some or i % 37 == 5 or i > 250:
                k[:, 0 if down else 1], c.tag[s] = 127 - far, 1
        c.c.ks[slots[280] // 16, 0, slots[280] % 16, 0] = ref.NONE
        q = c.q.double().numpy().reshape(n, 8, -1, 32)
        for i in range(n):
            low = 0 if down else 1
            q[i] *= 2.0 ** -17
            if i % 3 == 0:
                q[i, :, [g for g in range(D // 32) if g != low]] = 0.0
                q[i, :, low] *= 2.0 ** min(far, 30)
            elif i % 3 == 1:
                q[i, :, low] = 0.0
        c.q = torch.from_numpy(q.reshape(n, 8, D)).to(torch.float16)
        c.check(see=np.where(np.arange(n) % 3 == 0, 1 << 1, -1))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [8, 80])
@pytest.mark.parametrize("byte", [233, 241, 242, 246])
def test_the_largest_scales_of_k_with_one_that_is_not_a_number(n, byte, dtype):
    c = Case([31, n, byte], dtype, 8, 2, 64, length=[300], rows=[n], scale=2.0 ** (126 - byte), k_spread=0)
    t = np.arange(300)
    slots = c.table[0, t // 16] * 16 + t % 16
    for s in slots:
        c.c.ks[s // 16, :, s % 16] = byte
    c.tag[:], c.tag[slots[40]] = 2, 1
    c.c.ks[slots[40] // 16, 0, slots[40] % 16, 0] = ref.NONE
    c.check(see=np.where(np.arange(n) % 2 == 0, 3, 1 << 2))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("length", [1, 30, 300])
def test_the_smallest_scales_of_k_beyond_a_window(length, dtype):
    """Tokens behind the last one are in no window, whatever their bytes."""
    n = min(length, 5)
    c = Case([32, length], dtype, 8, 2, 64, length=[length], rows=[n], scale=2.0 ** 80, k_spread=0)
    c.c.ks[:] = 127
    t = np.arange(length)
    slots = c.table[0, t // 16] * 16 + t % 16
    for i, s in enumerate(slots):
        c.c.ks[s // 16, :, s % 16] = 47 if i % 3 else 27
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scales_of_k_all_over_their_range(dtype):
    """One token's scale in each window that there is; the scores of the largest ones decide."""
    c = Case([29], dtype, length=[64], rows=[5], scale=2.0 ** -115)
    t = np.arange(64)
    slots = c.table[0, t // 16] * 16 + t % 16
    for i, s in enumerate(slots):
        c.c.ks[s // 16, :, s % 16] = 27 + (i * 29) % 220
    c.check()


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


def test_the_same_bits_every_time():
    for kw in (dict(dtype="bf16", length=[5000], rows=[8]), dict(dtype="f16", D=64, length=[700, 40], rows=[50, 3])):
        c = Case(22, **kw)
        a = c.run()
        for _ in range(3):
            b = c.run()
            assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_layers_beyond_four_gibibytes():
    H, D, P = 8, 128, 64
    pages = (5 << 30) // (H * D * P // 2)
    c = Case(21, Hq=16, Hkv=H, D=D, P=P, length=[100], rows=[4])
    want, wlse = c.run()
    cfg = kv4.make_config("bf16", 16, H, D, c.scale, max_rows=4, page_tokens=P, n_phys_pages=pages, pages_per_request=2)
    bufs = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in kv4.cache_shapes(cfg)]
    table = [pages - 1, pages // 2]
    for at, page in zip(table, c.table[0]):
        for b, x in zip(bufs, c.c.pack()):
            b[0, at] = dev(x[page], torch.uint8).reshape(b.shape[2:])
    q = c.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(4, 16, device="cuda")
    h = kv4.PastaKv4(cfg, torch.empty(kv4.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"), page_table=dev([table]), k_codes=bufs[0],
                     v_codes=bufs[1], k_scale=bufs[2], v_scale=bufs[3], stream=torch.cuda.current_stream().cuda_stream)
    h.plan(dev([100]), dev([0, 4]), 4)
    h.attend(0, q, out, lse=lse)
    k, v = torch.empty(2, 3, H, D, device="cuda")
    h.read(0, dev([table[0] * P, table[0] * P + 63, table[1] * P + 20]), k, v)
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want) and np.array_equal(lse.double().cpu().numpy(), wlse)
    for got, full in zip((k, v), c.c.natural()):
        at = [c.table[0, 0] * P, c.table[0, 0] * P + 63, c.table[0, 1] * P + 20]
        assert np.array_equal(got.double().cpu().numpy(), full[at])
