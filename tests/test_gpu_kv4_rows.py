"""Rows into the 4-bit cache and out of it against the definition, row by row (codes, scales and values are exact: equal)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2502_11517_amd import kv4

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Cache:
    def __init__(self, H, D, P, pages, layers=1, seed=0, max_rows=1 << 14):
        self.H, self.D, self.P, self.pages = H, D, P, pages
        self.cfg = kv4.make_config("bf16", H, H, D, 1.0, n_layers=layers, max_rows=max_rows, page_tokens=P, n_phys_pages=pages)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.bufs = [torch.randint(0, 256, s, dtype=torch.uint8, device="cuda", generator=g) for s in kv4.cache_shapes(self.cfg)]
        self.h = kv4.PastaKv4(self.cfg, k_codes=self.bufs[0], v_codes=self.bufs[1], k_scale=self.bufs[2], v_scale=self.bufs[3],
                              stream=torch.cuda.current_stream().cuda_stream)
        self.want = [ref.Cache.unpack(pages, H, P, D, *(b[l].cpu().numpy() for b in self.bufs)) for l in range(layers)]

    def append(self, slot, k, v, layer=0):
        self.h.append(layer, torch.tensor(slot, dtype=torch.int32, device="cuda"), k, v)
        torch.cuda.synchronize()
        self.want[layer].append(slot, k.double().cpu().numpy(), v.double().cpu().numpy())

    def check(self):
        for l, w in enumerate(self.want):
            for got, want, name in zip(self.bufs, w.pack(), ("k", "v", "k_scale", "v_scale")):
                assert np.array_equal(got[l].cpu().numpy().reshape(want.shape), want), (l, name)

    def read(self, slot, dtype, layer=0):
        """(K, V) as read and as they should be"""
        n = len(slot)
        k, v = (torch.full((n, self.H, self.D), 7.0, dtype=TD[dtype], device="cuda") for _ in range(2))
        self.h.read(layer, torch.tensor(slot, dtype=torch.int32, device="cuda"), k, v)
        torch.cuda.synchronize()
        want = []
        for x in self.want[layer].natural():
            x = torch.from_numpy(x)
            row = torch.full((n, self.H, self.D), 7.0, dtype=torch.float64)
            for i, s in enumerate(slot):
                if 0 <= s < self.pages * self.P:
                    row[i] = x[s]
            want.append(row.to(TD[dtype]))
        return (k.cpu(), v.cpu()), want


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0))


def rows(seed, n, H, D, dtype, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, H, D, device="cuda", generator=g) * torch.exp(spread * torch.randn(n, H, D, device="cuda", generator=g))
    return x.to(TD[dtype])


def test_every_code_and_every_scale_read_back():
    """All 16 codes under all 256 scales, K and V, in the three types."""
    c = Cache(1, 64, 16, 32)
    for s in range(512):
        c.want[0].kc[s // 16, 0, s % 16] = np.arange(64) % 16
        c.want[0].vc[s // 16, 0, s % 16] = (np.arange(64) + s) % 16
        c.want[0].ks[s // 16, 0, s % 16] = [s % 256, (s + 128) % 256]
        c.want[0].vs[s // 16, 0, s % 16] = s % 256
    for b, w in zip(c.bufs, c.want[0].pack()):
        b.copy_(torch.from_numpy(np.ascontiguousarray(w)).reshape(b.shape))
    # scales that append does not give out (below 2^-100, above 2^119) are no part of the format
    out = [s for s in range(512) if all(27 <= x <= 246 or x == 255 for x in (s % 256, (s + 128) % 256))]
    for dtype in TD:
        got, want = c.read(out, dtype)
        assert same(got[0], want[0]) and same(got[1], want[1]), dtype


def test_values_next_to_a_rounding_border():
    """Every midpoint of two neighbouring codes, a bit of fp32 to either side, under several scales; the largest value beside them fixes the scale."""
    mids = (ref.LEVEL[:7] + ref.LEVEL[1:8]) / 2
    x = np.concatenate([[m, np.nextafter(np.float32(m), np.float32(9)), np.nextafter(np.float32(m), np.float32(-9))] for m in mids]).astype(np.float32)
    x = np.concatenate([x, ref.LEVEL[:8].astype(np.float32), [0.1, 0.2]])
    c = Cache(1, 64, 16, 4)
    for i, (scale, top) in enumerate([(1.0, 6.0), (2.0 ** -99, 7.0), (2.0 ** 118, 6.5), (2.0 ** 7, 5.0), (2.0 ** -9, 4.0), (1.0, 3.6)]):
        k = torch.zeros(1, 1, 64)
        k[0, 0, :31], k[0, 0, 32:63] = torch.from_numpy(x) * scale, torch.from_numpy(-x) * scale
        k[k.abs() > top * scale] = 0.0
        k[0, 0, 31], k[0, 0, 63] = top * scale, -top * scale
        c.append([3 + i], k.cuda(), k.flip(2).contiguous().cuda())
    c.check()


def test_the_scale_next_to_its_own_border():
    """7 * 2^e is the last value under 2^e."""
    c = Cache(2, 128, 16, 2)
    seven = np.float32(7.0)
    tops = [seven, np.nextafter(seven, np.float32(8)), np.nextafter(seven, np.float32(6)), np.float32(2.0 ** -140), np.float32(0.0), np.float32(3.4e38),
            np.float32(7.0 * 2.0 ** -100), np.float32(2.0 ** 122)]
    k = torch.zeros(len(tops), 2, 128)
    k[:, 0, 5] = torch.from_numpy(np.array(tops))
    k[:, 1, 127] = -k[:, 0, 5]
    c.append(list(range(8, 16)), k[:8].cuda(), k[:8].flip(0).contiguous().cuda())
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("H,D,P", [(1, 64, 16), (2, 128, 32), (3, 128, 64), (8, 64, 16), (5, 64, 32)])
def test_prompts_and_the_rows_behind_them(dtype, H, D, P):
    c = Cache(H, D, P, 12)
    table = np.random.default_rng(H).permutation(12)
    t = 0
    for i, n in enumerate([1, 1, 15, 3, 2 * P + 5, 1, 16, 1, 40]):
        at = np.arange(t, min(t + n, 12 * P))
        slot = table[at // P] * P + at % P
        c.append(slot, rows(i, len(at), H, D, dtype), rows(100 + i, len(at), H, D, dtype))
        t += n
    c.check()
    got, want = c.read(np.arange(12 * P), dtype)
    assert same(got[0], want[0]) and same(got[1], want[1])


@pytest.mark.parametrize("n", [1, 2, 16, 17, 31, 100, 333, 1400, 3000, 9000])
def test_calls_of_every_size(n):
    """Work-groups of 1 to 16 rows; runs that begin in one and end in the next."""
    c = Cache(2, 64, 16, -(-n // 16) + 3)
    perm = np.random.default_rng(n).permutation(c.pages)
    at = np.arange(5, 5 + n)
    slot = perm[at // 16] * 16 + at % 16
    k, v = rows(n, n, 2, 64, "bf16"), rows(n + 1, n, 2, 64, "bf16")
    c.append(slot, k, v)
    if n <= 400:
        c.check()
    got, want = c.read(slot, "f32")
    assert same(got[0], want[0]) and same(got[1], want[1])


def test_requests_that_write_single_rows_at_every_offset():
    c = Cache(3, 128, 16, 40)
    slot = [p * 16 + (5 * p) % 16 for p in range(40)]
    c.append(slot, rows(1, 40, 3, 128, "bf16"), rows(2, 40, 3, 128, "bf16"))
    c.append([p * 16 + (5 * p + 1) % 16 for p in range(40)], rows(3, 40, 3, 128, "bf16"), rows(4, 40, 3, 128, "bf16"))
    c.check()


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite(D):
    c = Cache(2, D, 16, 3)
    k, v = rows(5, 9, 2, D, "f32"), rows(6, 9, 2, D, "f32")
    k[1, 0, 3], k[2, 1, D - 1], k[3, 0, 0], v[4, 1, 7], v[5, 0, D - 1], v[6, 1, 0] = np.inf, np.nan, -np.inf, np.nan, np.inf, -np.inf
    k[7] = 0.0
    v[8] = -0.0
    c.append(list(range(20, 29)), k, v)
    c.check()
    got, want = c.read(list(range(16, 32)), "bf16")
    assert same(got[0], want[0]) and same(got[1], want[1]) and got[0].isnan().any() and got[1].isnan().any()


def test_slots_out_of_range_are_skipped():
    c = Cache(2, 64, 16, 4)
    slot = [3, -1, 21, 64, 33, 1 << 30, -(1 << 31), 55, 56, -1]  # (rows of one block are neighbours)
    c.append(slot, rows(7, 10, 2, 64, "bf16"), rows(8, 10, 2, 64, "bf16"))
    c.check()
    got, want = c.read(slot, "bf16")
    assert same(got[0], want[0]) and same(got[1], want[1])


def test_slots_may_be_read_in_any_order_and_twice():
    c = Cache(2, 128, 32, 4)
    c.append(list(range(32, 96)), rows(9, 64, 2, 128, "f16"), rows(10, 64, 2, 128, "f16"))
    slot = [33, 33, 32, 95, 94, 47, 48, 49, 50, 33, 64, 65, 66, 40, 41]
    got, want = c.read(slot, "f16")
    assert same(got[0], want[0]) and same(got[1], want[1])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_rows_apart_from_one_another(dtype, D):
    """Rows of a projection that holds q, k and v of a token side by side, and rows read into such."""
    H, n = 2, 21
    wide = rows(11, n, 1, 9 * D, dtype).view(n, 9, D)
    k, v = wide[:, 4:6], wide[:, 7:9]
    c = Cache(H, D, 16, 4)
    c.append(list(range(7, 7 + n)), k, v)
    c.check()
    out = torch.full((n, 7, D), 3.0, dtype=TD[dtype], device="cuda")
    c.h.read(0, torch.arange(7, 7 + n, dtype=torch.int32, device="cuda"), out[:, :2], out[:, 4:6])
    torch.cuda.synchronize()
    _, want = c.read(list(range(7, 7 + n)), dtype)
    assert same(out[:, :2].cpu(), want[0]) and same(out[:, 4:6].cpu(), want[1])
    assert (out[:, 2:4] == 3.0).all() and (out[:, 6:] == 3.0).all()


def test_one_of_the_two_alone():
    c = Cache(5, 64, 16, 2)
    slot = torch.arange(20, dtype=torch.int32, device="cuda")
    (k, v), _ = c.read(list(range(20)), "f32")
    for which in range(2):
        out = torch.zeros(20, 5, 64, device="cuda")
        c.h.read(0, slot, *((out, None) if which == 0 else (None, out)))
        torch.cuda.synchronize()
        assert same(out.cpu(), (k, v)[which])


def test_layers_are_apart():
    c = Cache(2, 64, 16, 3, layers=3)
    for l in (1, 0, 2):
        c.append([5, 6, 17 + l], rows(20 + l, 3, 2, 64, "bf16"), rows(30 + l, 3, 2, 64, "bf16"), layer=l)
    c.check()
    got, want = c.read([5, 6, 17, 18, 19], "bf16", layer=2)
    assert same(got[0], want[0]) and same(got[1], want[1])


def test_rows_behind_four_gibibytes_of_codes_and_of_rows():
    H, D, P = 8, 128, 64
    pages = (5 << 30) // (H * D * P // 2)
    cfg = kv4.make_config("bf16", H, H, D, 1.0, max_rows=64, page_tokens=P, n_phys_pages=pages)
    bufs = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in kv4.cache_shapes(cfg)]
    h = kv4.PastaKv4(cfg, k_codes=bufs[0], v_codes=bufs[1], k_scale=bufs[2], v_scale=bufs[3], stream=torch.cuda.current_stream().cuda_stream)
    n, far = 40, 1 << 26  # 40 rows 2^26 values apart
    slots = [pages * P - 40 + i for i in range(n)]
    slot = torch.tensor(slots, dtype=torch.int32, device="cuda")
    apart = torch.empty((n - 1) * far + H * D, dtype=torch.bfloat16, device="cuda").as_strided((n, H, D), (far, D, 1))
    k, v = rows(40, n, H, D, "bf16"), rows(41, n, H, D, "bf16")
    apart.copy_(k)
    h.append(0, slot, apart, v)
    small = Cache(H, D, P, 1)
    small.append([P - 40 + i for i in range(n)], k, v)
    (wk, wv), _ = small.read([P - 40 + i for i in range(n)], "bf16")
    apart.zero_()
    got = torch.zeros(n, H, D, dtype=torch.bfloat16, device="cuda")
    h.read(0, slot, apart, got)
    torch.cuda.synchronize()
    assert torch.equal(apart.cpu(), wk) and torch.equal(got.cpu(), wv)
    assert not bufs[0][0, :-1].any() and not bufs[3][0, :-1].any()


def test_captured_and_replayed():
    c = Cache(3, 64, 16, 4, max_rows=64)
    k, v, k2, v2 = (rows(i, 21, 3, 64, "bf16") for i in (50, 51, 52, 53))
    slots = list(range(7, 28))
    slot = torch.tensor(slots, dtype=torch.int32, device="cuda")
    ko, vo = torch.zeros(2, 21, 3, 64, device="cuda")
    stream = torch.cuda.Stream()
    h = kv4.PastaKv4(c.cfg, k_codes=c.bufs[0], v_codes=c.bufs[1], k_scale=c.bufs[2], v_scale=c.bufs[3], stream=stream.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        h.append(0, slot, k, v)
        h.read(0, slot, ko, vo)
    for i in range(4):
        if i == 2:
            k.copy_(k2), v.copy_(v2)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        c.want[0].append(slots, k.double().cpu().numpy(), v.double().cpu().numpy())
        c.check()
        for got, full in zip((ko, vo), c.want[0].natural()):
            assert torch.equal(got.double().cpu(), torch.from_numpy(np.ascontiguousarray(full[slots])))
