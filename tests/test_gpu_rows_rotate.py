"""Rotary positions against complex numbers in 64 bits.

Bound of an error, d that of a cosine or sine: eps / 2 |y| (the result's type) + d m (|x0| + |x1|), m the magnitude.
  fp32     the fraction of a turn is off by 2^-26, so the angle by 2 pi 2^-26 = 1.6 * 2^-24; the functions by 2 * 2^-24; m, the products, their sum by 2^-24 each: 2^-21
  16 bits  the hardware's functions are taken to be good to 2^-19
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2502_11517_amd import rows

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
OFF = {"f32": 2.0 ** -21, "bf16": 2.0 ** -19, "f16": 2.0 ** -19}


def turned(x, position, f, dims, layout, magnitude, backward):
    """(result, what its error's bound is measured by), float64"""
    angle = position.double()[:, None] * torch.tensor(f, dtype=torch.float64) * (-1 if backward else 1)
    z = torch.polar(torch.full_like(angle, magnitude), angle)[:, None]
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    a, b = (slice(0, dims // 2), slice(dims // 2, dims)) if layout == "half" else (slice(0, dims, 2), slice(1, dims, 2))
    w = torch.complex(x[..., a].double(), x[..., b].double()) * z
    y[..., a], y[..., b] = w.real, w.imag
    size[..., a] = size[..., b] = magnitude * (x[..., a].double().abs() + x[..., b].double().abs())
    return y, size


def check(got, x, position, f, dims, layout, magnitude, backward, dtype):
    want, size = turned(x.cpu(), position.cpu(), f, dims, layout, magnitude, backward)
    off = (got.cpu().double() - want).abs()
    bound = (torch.finfo(TD[dtype]).eps / 2 * want.abs() + OFF[dtype] * size) * (1 + 2.0 ** -7) + torch.finfo(TD[dtype]).smallest_normal
    assert (off <= bound).all(), float((off / bound).max())
    assert torch.equal(got[..., dims:], x[..., dims:])  # what is not turned stays


def make(seed, n, Hq, Hkv, D, dtype, far=50000):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k = (torch.randn(n, H, D, device="cuda", generator=g).to(TD[dtype]) for H in (Hq, Hkv))
    return q, k, torch.randint(0, far, (n,), device="cuda", generator=g, dtype=torch.int32)


def handle(Hq, Hkv, D, dims, layout, f, magnitude=1.0, max_rows=20000, stream=None):
    return rows.PastaRows(rows.make_config(max_rows=max_rows, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope_dims=dims, rope_layout=layout, rope_frequency=f,
                                           rope_magnitude=magnitude), stream=(stream or torch.cuda.current_stream()).cuda_stream)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,dims", [(128, 128), (64, 64), (128, 64), (128, 96), (128, 2), (64, 50), (64, 34), (8, 8), (256, 256), (96, 80), (256, 130), (16, 4)])
@pytest.mark.parametrize("Hq,Hkv,n", [(32, 8, 5), (3, 1, 33)])
def test_layouts_and_parts_of_heads(dtype, layout, D, dims, Hq, Hkv, n):
    f, _ = rows.rope_frequencies(dims)
    q, k, position = make(D + dims + n, n, Hq, Hkv, D, dtype)
    h = handle(Hq, Hkv, D, dims, layout, f)
    for backward in (False, True):
        qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
        h.rotate(position, q, qo, k, ko, backward=backward)
        torch.cuda.synchronize()
        check(qo, q, position, f, dims, layout, 1.0, backward, dtype)
        check(ko, k, position, f, dims, layout, 1.0, backward, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_far_positions_and_scaled_frequencies(dtype, scaling):
    f, m = rows.rope_frequencies(128, scaling=scaling, factor=1.0 if scaling == "none" else 32.0)
    q, k, _ = make(1, 9, 8, 2, 128, dtype)
    position = torch.tensor([0, 1, -1, 131071, 1 << 20, 1 << 24, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32, device="cuda")
    h = handle(8, 2, 128, 128, "half", f, m)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    h.rotate(position, q, qo, k, ko)
    torch.cuda.synchronize()
    check(qo, q, position, f, 128, "half", m, False, dtype)
    check(ko, k, position, f, 128, "half", m, False, dtype)
    if m == 1.0:
        assert torch.equal(qo[0], q[0]) and torch.equal(ko[0], k[0])


@pytest.mark.parametrize("n", [1, 2, 1000, 20000])
def test_calls_of_every_size(n):
    f, _ = rows.rope_frequencies(64)
    q, k, position = make(n, n, 4, 2, 64, "bf16")
    h = handle(4, 2, 64, 64, "interleaved", f)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    h.rotate(position, q, qo, k, ko)
    torch.cuda.synchronize()
    check(qo, q, position, f, 64, "interleaved", 1.0, False, "bf16")
    check(ko, k, position, f, 64, "interleaved", 1.0, False, "bf16")


@pytest.mark.parametrize("dims", [128, 64, 50])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_place_within_a_projection(dims, layout):
    """q and k as parts of rows that hold v, too: turned where they are, and nothing else is touched."""
    f, _ = rows.rope_frequencies(dims)
    n, Hq, Hkv, D = 21, 6, 2, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    qkv = torch.randn(n, Hq + 2 * Hkv, D, device="cuda", generator=g).bfloat16()
    before = qkv.clone()
    position = torch.arange(100, 100 + n, dtype=torch.int32, device="cuda")
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    handle(Hq, Hkv, D, dims, layout, f).rotate(position, q, q, k, k)
    torch.cuda.synchronize()
    check(qkv[:, :Hq], before[:, :Hq], position, f, dims, layout, 1.0, False, "bf16")
    check(qkv[:, Hq:Hq + Hkv], before[:, Hq:Hq + Hkv], position, f, dims, layout, 1.0, False, "bf16")
    assert torch.equal(qkv[:, Hq + Hkv:], before[:, Hq + Hkv:])


def test_one_of_the_two_alone():
    f, _ = rows.rope_frequencies(64)
    q, k, position = make(5, 7, 4, 2, 64, "f16")
    h = handle(4, 2, 64, 64, "half", f)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    h.rotate(position, q, qo)
    h.rotate(position, k=k, k_out=ko)
    torch.cuda.synchronize()
    check(qo, q, position, f, 64, "half", 1.0, False, "f16")
    check(ko, k, position, f, 64, "half", 1.0, False, "f16")


def test_the_way_back_is_the_gradient():
    """<g, R x> has the gradient R^T g; against differences of the call itself, in fp32: linear, so they are as good as its rounding."""
    n, H, D, dims = 3, 2, 16, 12
    f, _ = rows.rope_frequencies(dims)
    h = handle(H, 1, D, dims, "interleaved", f, 1.25)
    q, _, position = make(6, n, H, 1, D, "f32")
    g, _, _ = make(7, n, H, 1, D, "f32")
    call = lambda x, **kw: (o := torch.empty_like(x), h.rotate(position, x, o, **kw))[0]  # noqa: E731
    grad = call(g, backward=True).double()
    for i, j, d in ((0, 0, 0), (1, 1, 5), (2, 0, 11), (0, 1, 15), (2, 1, 6)):
        up, down = q.clone(), q.clone()
        up[i, j, d] += 1.0
        down[i, j, d] -= 1.0
        step = float(((call(up).double() - call(down).double()) * g.double()).sum() / 2)
        # every value of a plane is off by 2^-21 (|x0| + |x1|) m, |x| < 8 and |g| < 5 here
        assert abs(step - float(grad[i, j, d])) < 2 * 2 * 2.0 ** -21 * 16 * 1.25 * 5


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_values_that_are_not_finite_stay_in_their_planes(layout):
    f, _ = rows.rope_frequencies(64)
    q, k, position = make(8, 4, 2, 1, 64, "bf16")
    q[1, 0, 5], q[2, 1, 40] = float("nan"), float("inf")
    qo = torch.empty_like(q)
    handle(2, 1, 64, 64, layout, f).rotate(position, q, qo)
    torch.cuda.synchronize()
    bad = ~qo.isfinite()
    want = torch.zeros_like(bad)
    for i, j, d in ((1, 0, 5), (2, 1, 40)):
        other = (d + 32) % 64 if layout == "half" else d ^ 1
        want[i, j, [d, other]] = True
    assert torch.equal(bad, want)


def test_captured_and_replayed_on_another_stream():
    f, _ = rows.rope_frequencies(128)
    q, k, position = make(9, 8, 32, 8, 128, "bf16")
    s = torch.cuda.Stream()
    h = handle(32, 8, 128, 128, "half", f, stream=s)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        h.rotate(position, q, qo, k, ko)
    for i in range(4):
        position.fill_(1000 * i + 7)
        qo.zero_(), ko.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(qo, q, position, f, 128, "half", 1.0, False, "bf16")
        check(ko, k, position, f, 128, "half", 1.0, False, "bf16")


def test_the_cpu_reference_is_a_rotation():
    x = torch.randn(2, 1, 8)
    y, _ = turned(x, torch.tensor([3, 5]), [1.0, 0.5], 4, "half", 1.0, False)
    assert np.isclose(float(y[0, 0, 0]), float(x[0, 0, 0] * np.cos(3.0) - x[0, 0, 2] * np.sin(3.0)), atol=1e-6)


def test_rows_that_lie_far_apart():
    """Offsets beyond 2^31 values, in place, beside rows that lie side by side."""
    f, _ = rows.rope_frequencies(64)
    q, k, position = make(10, 40, 4, 2, 64, "bf16")
    far = 1 << 26
    apart = torch.empty(39 * far + 4 * 64, dtype=torch.bfloat16, device="cuda").as_strided((40, 4, 64), (far, 64, 1))
    apart.copy_(q)
    h = handle(4, 2, 64, 64, "half", f, max_rows=40)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    h.rotate(position, q, qo, k, ko)
    h.rotate(position, apart, apart, k, ko)
    torch.cuda.synchronize()
    assert torch.equal(apart.cpu(), qo.cpu())
