"""Attention over the 4-bit cache with at most 16 stacked rows in a unit: one or a few threads, against the 64-bit form.  Bounds are test_gpu_kv4_attend's."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2502_11517_amd import kv4
from test_gpu_kv4_attend import Case

pytestmark = pytest.mark.gpu

# (dtype, D, Hq, Hkv, rows): 16 stacked rows, fewer, and one more than there is room for
FEW = [("bf16", 128, 8, 2, 4), ("f16", 128, 6, 6, 16), ("f16", 64, 4, 2, 8), ("bf16", 64, 16, 2, 2), ("f16", 128, 16, 2, 1), ("bf16", 64, 3, 3, 5), ("f16", 64, 8, 8, 17)]


@pytest.mark.parametrize("dtype,D,Hq,Hkv,n", FEW)
@pytest.mark.parametrize("T", [17, 48, 63, 64, 65, 128, 193, 255, 256, 257, 320, 767, 1023, 1024, 1025, 3000])
def test_lengths_around_a_step(dtype, D, Hq, Hkv, n, T):
    n = min(n, T)
    c = Case([n, T, 41], dtype, Hq, Hkv, D, 16 if T % 2 else 64, [T], [n])
    c.check()
    see = c.rng.integers(-2 ** 63, 2 ** 63, n)
    see[n // 2] = 0
    c.check(see=see, prefix=[T // 3], cap=15.0 if T % 3 else 0.0, slopes=c.rng.uniform(0.0, 0.02, Hq).astype(np.float32),
            row_position=c.rng.integers(0, 5000, n) if T % 2 else None)


@pytest.mark.parametrize("table", [None, 400])  # (in a wide table tokens are split)
def test_few_rows_beside_many(table):
    length, rows = [700, 700, 64, 1, 900, 300, 5000], [4, 5, 1, 1, 25, 0, 2]
    c = Case(42, length=length, rows=rows, width=table, pad=3)
    c.check()
    c.check(see=c.rng.integers(-2 ** 63, 2 ** 63, c.n), prefix=[600, 0, 64, 1, 100, 7, 4000])


@pytest.mark.parametrize("dtype,spread", [("bf16", 3), ("f16", 3), ("bf16", 9), ("f16", 9), ("bf16", 30)])  # (fp16 ends at 2^16)
@pytest.mark.parametrize("D", [64, 128])
def test_scales_of_v_apart(dtype, D, spread):
    for n in (1, 4):
        Case([n, 43, spread], dtype, 8, 2, D, length=[333], rows=[n], spread=spread).check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("far", [12, 13, 14, 20, 34])
@pytest.mark.parametrize("down", [False, True])
def test_scales_of_k_beyond_a_window(D, far, down):
    """As test_scales_of_k_beyond_a_window_of_fp16: rows 0 and 3 see tokens alone whose group of dims is at 2^-far, in sizes that make scores of 1."""
    c = Case([44, D, far, down], "f16", 8, 2, D, length=[300], rows=[4], scale=2.0 ** 14, k_spread=0)
    t = np.arange(300)
    slots = c.table[0, t // 16] * 16 + t % 16
    c.tag[:] = 2
    low = 0 if down else 1
    for i, s in enumerate(slots):
        k = c.c.ks[s // 16, :, s % 16]
        k[:] = 127
        if i % 37 == 5 or i > 250:
            k[:, low], c.tag[s] = 127 - far, 1
    q = c.q.double().numpy().reshape(4, 8, -1, 32) * 2.0 ** -17
    for i in (0, 3):
        q[i, :, [g for g in range(D // 32) if g != low]] = 0.0
        q[i, :, low] *= 2.0 ** min(far, 30)
    q[1, :, low] = 0.0
    c.q = torch.from_numpy(q.reshape(4, 8, D)).to(torch.float16)
    c.check(see=np.array([1 << 1, -1, -1, 1 << 1]))


@pytest.mark.parametrize("D", [64, 128])
def test_scales_of_k_and_v_that_are_not_numbers(D):
    for dtype in ("bf16", "f16"):
        c = Case([45, D], dtype, 8, 2, D, length=[200], rows=[4])
        c.tag[:] = 0
        slots = [c.table[0, t // 16] * 16 + t % 16 for t in (0, 49, 66)]
        c.tag[slots] = 9
        c.c.ks[slots[0] // 16, 0, slots[0] % 16, D // 32 - 1] = c.c.ks[slots[1] // 16, 1, slots[1] % 16, 0] = ref.NONE
        c.c.vs[slots[2] // 16, 1, slots[2] % 16] = ref.NONE
        see = np.array([1, 1 | 1 << 9, 1 << 9, 1])
        out, lse = c.run(see=see)
        want, wlse = c.want(see=see)[:2]
        assert np.array_equal(np.isnan(lse), np.isnan(wlse)) and np.array_equal(np.isnan(out), np.isnan(want))
        assert np.isnan(out[1:3]).any() and not np.isnan(out[[0, 3]]).any()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f16", 128)])
def test_units_longer_than_a_waves_list_of_blocks(dtype, D):
    """5000 tokens and more to a unit (a wave lists 16 steps of 64 tokens at a time): 64 kv heads leave eight units to the chip."""
    H, T, n, P = 64, 43000 if D == 64 else 41000, 2, 16
    td = torch.bfloat16 if dtype == "bf16" else torch.float16
    g = torch.Generator(device="cuda").manual_seed(46)
    pages = -(-T // P)
    cfg = kv4.make_config(dtype, H, H, D, D ** -0.5, max_requests=1, max_rows=n, page_tokens=P, n_phys_pages=pages, pages_per_request=pages)
    k, v = (torch.randint(0, 16, (pages, H, P, D), device="cuda", generator=g, dtype=torch.uint8) for _ in range(2))
    ks = torch.randint(125, 128, (pages, H, P, D // 32), device="cuda", generator=g, dtype=torch.uint8)
    vs = torch.randint(125, 128, (pages, H, P), device="cuda", generator=g, dtype=torch.uint8)
    pack = lambda x: (x[..., 0::2] | x[..., 1::2] << 4).contiguous()  # noqa: E731
    shapes = kv4.cache_shapes(cfg)
    bufs = [pack(k.view(pages, H, P, D // 32, 32).transpose(2, 3)).view(shapes[0]), pack(v.transpose(2, 3)).view(shapes[1]), ks.view(shapes[2]), vs.view(shapes[3])]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.randn(n, H, D, device="cuda", generator=g).to(td)
    out, lse = torch.empty_like(q), torch.empty(n, H, device="cuda")
    ws = torch.empty(kv4.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    h = kv4.PastaKv4(cfg, ws, page_table=torch.arange(pages, device="cuda", dtype=torch.int32).view(1, -1), k_codes=bufs[0], v_codes=bufs[1], k_scale=bufs[2],
                     v_scale=bufs[3], stream=torch.cuda.current_stream().cuda_stream)
    h.plan(i32([T]), i32([0, n]), n)
    h.attend(0, q, out, lse=lse)
    torch.cuda.synchronize()
    level = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    for head in range(0, H, 9):
        kk = (level[k[:, head].long()].view(pages, P, D // 32, 32) * torch.exp2(ks[:, head].double() - 127)[..., None]).reshape(-1, D)[:T]
        vv = (level[v[:, head].long()] * torch.exp2(vs[:, head].double() - 127)[..., None]).reshape(-1, D)[:T]
        s = (q[:, head].double() @ kk.T) * D ** -0.5
        s[0, T - 1] = -torch.inf
        w, want_lse = torch.softmax(s, -1), torch.logsumexp(s, -1)
        want, mean = w @ vv, w @ vv.abs()
        most_s = (q[:, head].double().abs() @ kk.abs().T).amax(-1) * D ** -0.5
        ds = 2.0 ** -20 * (1 + most_s)
        # half a step of the result; weights' rounding to fp16 and the scores' error, over the mean magnitude; what fp16 does not hold of each weight
        bound = torch.finfo(td).eps / 2 * want.abs() + (2.0 ** -11 + 2 * ds[:, None]) * mean + T * 2.0 ** -25 * vv.abs().max() * w.amax(-1, keepdim=True)
        assert ((out[:, head].double() - want).abs() <= bound * (1 + 2.0 ** -6)).all()
        assert ((lse[:, head].double() - want_lse).abs() <= ds + 2.0 ** -20 * want_lse.abs()).all()


def test_pages_and_requests_that_are_not_there():
    c = Case(47, length=[200, 40, 90], rows=[3, 4, 2], pad=4)
    c.table[0, 2], c.table[0, 3], c.table[0, 9], c.table[1, 2] = -1, 1 << 29, c.pages, -(1 << 31)
    c.check()
    c.check(see=c.rng.integers(-2 ** 63, 2 ** 63, c.n), prefix=[50, 0, 90])
    c.table[1, :] = -1
    slot = np.zeros(c.n, int)
    slot[7:9] = -1  # request 2 was refused
    out, lse = c.check(slot=slot, refused=(2,), see=np.full(c.n, -1))
    assert (out[3:] == 0).all() and np.isneginf(lse[3:]).all()
    c.length, c.offs = np.array([1 << 30, -9, 90]), np.array([-5, 4, 2, 1 << 20])
    c.run()


def test_the_same_bits_every_time():
    for kw in (dict(dtype="bf16", length=[5000], rows=[3]), dict(dtype="f16", D=64, length=[700, 40], rows=[4, 1])):
        c = Case(48, **kw)
        a = c.run()
        for _ in range(3):
            b = c.run()
            assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_two_captured_steps_at_a_time():
    """Each with a handle and a workspace of its own over one cache, replayed side by side on two streams: what they read they share, what they write they do not."""
    cases = [Case(49, length=[3000], rows=[n]) for n in (4, 20)]
    a = cases[0]
    cases[1].c, cases[1].table, cases[1].pages = a.c, a.table, a.pages
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    bufs = [torch.from_numpy(np.ascontiguousarray(b)).to("cuda", torch.uint8).reshape(s) for b, s in zip(a.c.pack(), kv4.cache_shapes(a.config()))]
    table = i32(a.table)
    steps = []
    for c in cases:
        cfg, stream = c.config(), torch.cuda.Stream()
        ws = torch.empty(kv4.query_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        q = c.q.cuda()
        out, lse = torch.zeros_like(q), torch.zeros(c.n, c.Hq, device="cuda")
        h = kv4.PastaKv4(cfg, ws, page_table=table, k_codes=bufs[0], v_codes=bufs[1], k_scale=bufs[2], v_scale=bufs[3], stream=stream.cuda_stream)
        length, offs = i32(c.length), i32(c.offs)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            h.plan(length, offs, c.n)
            for _ in range(4):
                h.attend(0, q, out, lse=lse)
        steps.append((c, stream, graph, out, lse, (h, ws, q, length, offs)))
    want = [c.run() for c in cases]
    for i in range(5):
        for c, stream, graph, out, lse, _ in steps:
            with torch.cuda.stream(stream):
                out.zero_(), lse.zero_()
                graph.replay()
        if i % 2:
            (torch.ones(100, device="cuda") * i).sum().item()
        torch.cuda.synchronize()
        for (c, _, _, out, lse, _), (o, l) in zip(steps, want):
            assert np.array_equal(out.double().cpu().numpy(), o) and np.array_equal(lse.double().cpu().numpy(), l)
