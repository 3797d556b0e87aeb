"""Rows into the 8-bit cache against the walk block by block (codes and scales are exact: equal)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv8_ref as ref
from paper_2502_11517_amd import kv8

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Cache:
    def __init__(self, codes, H, D, P, pages, seed=0, dtype="bf16", max_rows=1 << 14, blank=0x55):
        self.codes, self.H, self.D, self.P, self.pages = codes, H, D, P, pages
        self.cfg = kv8.make_config(codes, "bf16", H, H, D, 1.0, max_rows=max_rows, page_tokens=P, n_phys_pages=pages)
        ks, vs, ss = kv8.cache_shapes(self.cfg)
        self.k = torch.full(ks, blank, dtype=torch.uint8, device="cuda")
        self.v = torch.full(vs, blank, dtype=torch.uint8, device="cuda")
        self.ks = torch.full(ss, 123.0, device="cuda")
        self.vs = torch.full(ss, 123.0, device="cuda")
        self.h = kv8.PastaKv8(self.cfg, torch.empty(kv8.query_workspace_bytes(self.cfg), dtype=torch.uint8, device="cuda"), k_codes=self.k,
                              v_codes=self.v, k_scale=self.ks, v_scale=self.vs, stream=torch.cuda.current_stream().cuda_stream)
        values = ref.code_values(codes)
        self.want = [values[ref.k_natural(self.k.cpu().numpy()[0])], self.ks.cpu().numpy()[0].astype(float),
                     values[np.moveaxis(self.v.cpu().numpy()[0], -1, -2)], self.vs.cpu().numpy()[0].astype(float)]

    def append(self, slot, k, v):
        self.h.append(0, torch.tensor(slot, dtype=torch.int32, device="cuda"), k, v)
        torch.cuda.synchronize()
        kf, vf = k.double().cpu().numpy(), v.double().cpu().numpy()
        ref.append(self.codes, self.want[0], self.want[1], kf, slot, self.P)
        ref.append(self.codes, self.want[2], self.want[3], vf, slot, self.P)

    def check(self):
        values = ref.code_values(self.codes)
        got = [values[ref.k_natural(self.k.cpu().numpy()[0])], self.ks.cpu().numpy()[0], values[np.moveaxis(self.v.cpu().numpy()[0], -1, -2)],
               self.vs.cpu().numpy()[0]]
        for g, w, name in zip(got, self.want, ("k", "k_scale", "v", "v_scale")):
            same = np.array_equal(g.astype(float), w, equal_nan=True)
            assert same, name


def rows(seed, n, H, D, dtype, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, H, D, device="cuda", generator=g) * torch.exp(spread * torch.randn(n, H, 1, device="cuda", generator=g))
    return x.to(TD[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("H,D,P", [(1, 64, 16), (2, 128, 32), (3, 128, 64), (8, 64, 16)])
def test_prompts_and_the_rows_behind_them(codes, dtype, H, D, P):
    c = Cache(codes, H, D, P, 12, dtype=dtype)
    table = np.random.default_rng(H).permutation(12)
    t = 0
    for i, n in enumerate([1, 1, 15, 3, 2 * P + 5, 1, 16, 1, 40]):
        at = np.arange(t, min(t + n, 12 * P))
        slot = table[at // P] * P + at % P
        c.append(slot, rows(i, len(at), H, D, dtype), rows(100 + i, len(at), H, D, dtype))
        t += n
    c.check()


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_single_rows_whose_size_grows_and_falls(codes):
    c = Cache(codes, 2, 64, 16, 4)
    size = [1, 1.01, 3, 1e-3, 100, 99, 0, 1e4, 1e-30, 2e4, 3e38, 1, 1e30, 0, 5, 6]
    for t, s in enumerate(size):
        x, y = rows(t, 1, 2, 64, "f32", 0.0) * s, rows(50 + t, 1, 2, 64, "f32", 0.0) / max(s, 1e-30)
        c.append([16 + t], x, y)
        c.check()


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_values_next_to_a_rounding_border(codes):
    """Every midpoint of two neighbouring codes, a bit of fp32 to either side, at several scales."""
    v = np.unique(np.abs(ref.code_values(codes)[~np.isnan(ref.code_values(codes))]))
    v = v[v <= ref.TOP[codes]]
    mid = ((v[1:] + v[:-1]) / 2).astype(np.float32)
    x = np.concatenate([mid, np.nextafter(mid, np.float32(np.inf)), np.nextafter(mid, np.float32(0)), v.astype(np.float32)])
    x = np.concatenate([x, -x])
    for e in (-20, 0, 7):
        n = -(-len(x) // 63)
        full = np.zeros((n, 1, 64), np.float32)
        full[:, 0, 0] = ref.TOP[codes]
        flat = np.zeros(n * 63, np.float32)
        flat[:len(x)] = x
        full[:, 0, 1:] = flat.reshape(n, 63)
        rows_ = torch.from_numpy(full * np.float32(2.0 ** e)).cuda()
        c = Cache(codes, 1, 64, 16, 4)
        c.append(np.arange(n), rows_, -rows_)
        c.check()
        assert (c.want[1][0, 0, 0] == 2.0 ** e)


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
def test_a_largest_value_next_to_where_the_scale_doubles(codes):
    for x in (ref.TOP[codes], np.nextafter(np.float32(ref.TOP[codes]), np.float32(np.inf)), np.nextafter(np.float32(ref.TOP[codes]), np.float32(0)),
              np.float32(2.0 ** -126), np.float32(1e-45), np.finfo(np.float32).max):
        c = Cache(codes, 1, 64, 16, 1)
        r = torch.zeros(2, 1, 64, device="cuda")
        r[1, 0, 5] = float(x)
        c.append([0, 1], r, -r)
        c.check()


@pytest.mark.parametrize("codes", ["e4m3", "int8"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_what_is_not_finite_makes_its_block_nan_until_it_is_started_anew(codes, bad):
    c = Cache(codes, 3, 128, 16, 3)
    c.append(np.arange(20), rows(1, 20, 3, 128, "bf16"), rows(2, 20, 3, 128, "bf16"))
    k, v = rows(3, 2, 3, 128, "bf16"), rows(4, 2, 3, 128, "bf16")
    k[1, 1, 77] = bad
    v[0, 2, 3] = bad
    c.append([20, 21], k, v)
    c.check()
    assert np.isnan(c.want[1]).sum() == 1 and np.isnan(c.want[3]).sum() == 1
    c.append([22], rows(5, 1, 3, 128, "bf16"), rows(6, 1, 3, 128, "bf16"))
    c.check()
    c.append([16], rows(7, 1, 3, 128, "bf16"), rows(8, 1, 3, 128, "bf16"))
    c.check()
    assert not np.isnan(c.want[1]).any()
    values = {0x7f, 0xff} if codes == "e4m3" else set()
    assert not values & set(np.unique(c.k.cpu().numpy())) and not values & set(np.unique(c.v.cpu().numpy()))


def test_rows_without_a_slot_are_skipped():
    c = Cache("e4m3", 2, 64, 16, 3)
    slot = [-1, 16, 17, 18, -1, 48, 1 << 30, 0, -5]
    c.append(slot, rows(1, 9, 2, 64, "bf16"), rows(2, 9, 2, 64, "bf16"))
    c.check()


@pytest.mark.parametrize("n", [1024, 1025, 2000])
def test_many_rows_in_one_call(n):
    """Both sides of where a work-group looks at 16 rows; runs that cross its border, and single rows of many blocks."""
    rng = np.random.default_rng(n)
    c = Cache("int8", 2, 64, 32, 400)
    slot, used = [], rng.permutation(400 * 2)
    for b in used:
        o, m = int(rng.integers(0, 16)), int(rng.integers(1, 17))
        slot += [int(b) * 16 + t for t in range(o, min(16, o + m))]
        if len(slot) >= n:
            break
    slot = slot[:n]
    c.append(slot, rows(1, n, 2, 64, "bf16"), rows(2, n, 2, 64, "bf16"))
    c.check()


def test_layers_beyond_four_gibibytes():
    """Pages at both ends of a cache whose codes pass 32-bit offsets."""
    H, D, P = 8, 128, 64
    pages = (5 << 30) // (H * D * P)
    c = kv8.make_config("e4m3", "bf16", H, H, D, 1.0, max_rows=64, page_tokens=P, n_phys_pages=pages)
    ks, vs, ss = kv8.cache_shapes(c)
    k, v = torch.zeros(ks, dtype=torch.uint8, device="cuda"), torch.zeros(vs, dtype=torch.uint8, device="cuda")
    s, t = torch.zeros(ss, device="cuda"), torch.zeros(ss, device="cuda")
    h = kv8.PastaKv8(c, torch.empty(kv8.query_workspace_bytes(c), dtype=torch.uint8, device="cuda"), k_codes=k, v_codes=v, k_scale=s, v_scale=t,
                     stream=torch.cuda.current_stream().cuda_stream)
    small = Cache("e4m3", H, D, P, 2, blank=0)
    at = [0, pages - 1]
    slot = np.concatenate([np.arange(20), P + 16 + np.arange(20)])
    far = np.concatenate([np.arange(20), (pages - 1) * P + 16 + np.arange(20)])
    x, y = rows(1, 40, H, D, "bf16"), rows(2, 40, H, D, "bf16")
    small.append(slot, x, y)
    small.check()
    h.append(0, torch.tensor(far, dtype=torch.int32, device="cuda"), x, y)
    torch.cuda.synchronize()
    assert torch.equal(k[0][at], small.k[0]) and torch.equal(v[0][at], small.v[0])
    assert int(k[0].count_nonzero()) == int(small.k.count_nonzero()) and int(s.count_nonzero()) == 4 * H
