"""The library of a step's rows on the CPU: exported symbols, refusals of arguments, sizes, frequencies.  No call here reaches a launch."""
from __future__ import annotations

import ctypes as C
import math
import os
import re
import struct
import subprocess

import pytest
import torch

from paper_2502_11517_amd import rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # an aligned address that is never read


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(rows.library_path()):
        rows.build_library()


ROPE = dict(max_rows=64, n_q_heads=32, n_kv_heads=8, head_dim=128, rope_dims=128, rope_layout="half", rope_frequency=FAKE)
VERIFY = dict(max_rows=64, vocab=100000, max_sequences=16)


def rotates(**kw):
    return rows.PastaRows(rows.make_config(**{**ROPE, **kw}))


def verifies(workspace=FAKE, **kw):
    return rows.PastaRows(rows.make_config(**{**VERIFY, **kw}), workspace, workspace_bytes=1 << 40)


def test_every_declared_symbol_is_exported():
    hdr = open(os.path.join(ROOT, "include", "pasta_rows.h")).read()
    declared = set(re.findall(r"\bint32_t\s+(pasta_rows_\w+)\s*\(", hdr))
    assert declared == {"pasta_rows_" + n for n in ("create", "destroy", "rotate", "verify")}
    syms = subprocess.run(["nm", "-D", "--defined-only", rows.library_path()], capture_output=True, text=True).stdout
    assert declared <= {l.split()[-1] for l in syms.splitlines() if " T " in l}


@pytest.mark.parametrize("kw", [dict(max_rows=0), dict(max_rows=1 << 24), dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_q_heads=1000, n_kv_heads=25), dict(head_dim=0), dict(head_dim=12),
                                dict(head_dim=264, rope_dims=8), dict(rope_dims=130), dict(rope_dims=7), dict(rope_dims=-2), dict(rope_layout=2),
                                dict(rope_magnitude=float("nan")), dict(rope_magnitude=float("inf")), dict(max_sequences=4)])
def test_configurations_of_rotate_that_are_refused(kw):
    with pytest.raises(rows.PastaError) as e:
        rows.query_workspace_bytes(rows.make_config(**{**ROPE, **kw}))
    assert e.value.code == rows.E_INVAL


@pytest.mark.parametrize("kw", [dict(max_rows=0), dict(max_rows=1 << 24), dict(vocab=-1), dict(vocab=(1 << 22) + 1), dict(max_sequences=0), dict(max_sequences=65536), dict(vocab=0),
                                dict(head_dim=64), dict(n_q_heads=1)])
def test_configurations_of_verify_that_are_refused(kw):
    with pytest.raises(rows.PastaError) as e:
        rows.query_workspace_bytes(rows.make_config(**{**VERIFY, **kw}))
    assert e.value.code == rows.E_INVAL


def test_workspaces_and_addresses():
    assert rows.query_workspace_bytes(rows.make_config(**ROPE)) == 0
    assert rows.query_workspace_bytes(rows.make_config(**{**VERIFY, "vocab": 32768})) == 0
    size = rows.query_workspace_bytes(rows.make_config(**VERIFY))
    assert size == 16 * (98 * 8 + 8)
    for ws, n, code in ((FAKE, size - 1, rows.E_CAPACITY), (FAKE + 16, size, rows.E_INVAL)):
        with pytest.raises(rows.PastaError) as e:
            rows.PastaRows(rows.make_config(**VERIFY), ws, workspace_bytes=n)
        assert e.value.code == code
    with pytest.raises(rows.PastaError):
        rotates(rope_frequency=FAKE + 4)


def test_rotate_refusals():
    h = rotates()
    good = dict(position=FAKE, q=FAKE, q_out=FAKE, k=FAKE, k_out=FAKE, n_rows=4, dtype="bf16")
    for kw, code in ((dict(n_rows=-1), rows.E_INVAL), (dict(n_rows=65), rows.E_CAPACITY), (dict(dtype=3), rows.E_INVAL), (dict(position=None), rows.E_INVAL),
                     (dict(position=FAKE + 2), rows.E_INVAL), (dict(q=None), rows.E_INVAL), (dict(k_out=None), rows.E_INVAL), (dict(q=FAKE + 8), rows.E_INVAL),
                     (dict(k_out=FAKE + 4), rows.E_INVAL), (dict(q=None, q_out=None, k=None, k_out=None), rows.E_INVAL), (dict(n_rows=0), rows.OK),
                     (dict(n_rows=0, position=None, q=None, q_out=None), rows.OK)):
        assert h.prepare_rotate(**{**good, **kw})() == code, kw
    assert rotates(rope_frequency=None).prepare_rotate(**good)() == rows.E_INVAL
    assert verifies().prepare_rotate(**good)() == rows.E_INVAL  # a handle for verify
    for field, value in (("q_stride", 100), ("q_stride", 4096 + 4), ("k_stride", 1016), ("q_out_stride", -4096), ("k_out_stride", 1 << 50), ("q_stride", 8192)):
        a = rows.RotateArgs(C.sizeof(rows.RotateArgs), 0, 4, rows.BF16, FAKE, FAKE, FAKE, FAKE, FAKE)
        setattr(a, field, value)  # (the last one: in place, with another stride)
        assert rows.load_library().pasta_rows_rotate(h._h, C.byref(a)) == rows.E_INVAL, field


def test_verify_refusals():
    h = verifies()
    good = dict(row_offsets=FAKE, token=FAKE, target=FAKE, draw=FAKE, last_draw=FAKE, accepted=FAKE, next_token=FAKE, draft=FAKE, length=FAKE, keep=FAKE,
                row_position=FAKE, position_out=FAKE, n_sequences=4, n_rows=9, dtype="f32")
    for kw, code in ((dict(n_rows=-1), rows.E_INVAL), (dict(n_rows=65), rows.E_CAPACITY), (dict(n_sequences=-1), rows.E_INVAL),
                     (dict(n_sequences=17), rows.E_CAPACITY), (dict(dtype=9), rows.E_INVAL), (dict(row_offsets=None), rows.E_INVAL), (dict(token=None), rows.E_INVAL),
                     (dict(target=None), rows.E_INVAL), (dict(draw=None), rows.E_INVAL), (dict(last_draw=None), rows.E_INVAL), (dict(accepted=None), rows.E_INVAL),
                     (dict(next_token=None), rows.E_INVAL), (dict(length=None), rows.E_INVAL), (dict(keep=None), rows.E_INVAL),
                     (dict(row_position=None), rows.E_INVAL), (dict(position_out=None), rows.E_INVAL), (dict(target=FAKE + 2), rows.E_INVAL),
                     (dict(draft=FAKE + 1, dtype="bf16"), rows.E_INVAL), (dict(accepted=FAKE + 2), rows.E_INVAL), (dict(slot=FAKE + 1), rows.E_INVAL), (dict(n_sequences=0), rows.OK)):
        assert h.prepare_verify(**{**good, **kw})() == code, kw
    assert verifies(workspace=None).prepare_verify(**good)() == rows.E_INVAL
    assert rotates().prepare_verify(**good)() == rows.E_INVAL  # a handle for rotate
    for field, value in (("target_stride", 99999), ("draft_stride", -100000), ("target_stride", 1 << 41)):
        a = rows.VerifyArgs(C.sizeof(rows.VerifyArgs), 0, 4, 9, rows.F32, *[FAKE] * 5, 0, 0, *[FAKE] * 8)
        setattr(a, field, value)
        assert rows.load_library().pasta_rows_verify(h._h, C.byref(a)) == rows.E_INVAL, field


def test_destroyed_handles_and_wrong_structs():
    h = rotates()
    lib = rows.load_library()
    for name, args in (("rotate", rows.RotateArgs), ("verify", rows.VerifyArgs)):
        f = getattr(lib, "pasta_rows_" + name)
        assert f(h._h, C.byref(args(4))) == rows.E_INVAL and f(h._h, C.byref(args(C.sizeof(args), 2))) == rows.E_INVAL
        assert f(None, C.byref(args(C.sizeof(args)))) == rows.E_STATE and f(h._h, None) == rows.E_INVAL
    call = h.prepare_rotate(FAKE, FAKE, FAKE, n_rows=4, dtype="bf16")
    h.destroy()
    assert call() == rows.E_STATE and lib.pasta_rows_destroy(None) == rows.OK


def test_tensors_are_checked():
    h, v = rotates(), verifies()
    q = torch.zeros(8, 32, 128)
    for x in (q.bfloat16(), q[:4], q[:, ::2], q[:, :, ::2], q.transpose(0, 1), q[:1].expand(8, 32, 128), q):
        with pytest.raises(ValueError):  # (the last one: host memory)
            h.prepare_rotate(FAKE, x, q, n_rows=8, dtype="f32")
    p = torch.zeros(9, 100032)
    for x in (p.half(), p[:8], p[:, :99999], p[:, ::2], p[:1].expand(9, 100032), p):
        with pytest.raises(ValueError):
            v.prepare_verify(FAKE, FAKE, x, FAKE, FAKE, FAKE, FAKE, n_sequences=2, n_rows=9, dtype="f32")
    with pytest.raises(ValueError):
        rotates(rope_frequency=torch.zeros(63, dtype=torch.float64))
    with pytest.raises(ValueError):
        rotates(rope_frequency=torch.zeros(64, dtype=torch.float64))  # host memory


def test_frequencies():
    f, m = rows.rope_frequencies(128, 10000.0)
    assert m == 1.0 and len(f) == 64 and f[0] == 1.0 and math.isclose(f[63], 10000.0 ** (-126 / 128), rel_tol=1e-15)
    assert rows.rope_frequencies(128, scaling="linear", factor=8.0)[0] == [x / 8.0 for x in f]
    g, _ = rows.rope_frequencies(128, scaling="base", factor=8.0)
    assert g[0] == 1.0 and math.isclose(g[63], f[63] / 8.0, rel_tol=1e-12) and all(a <= b for a, b in zip(g, f))
    assert rows.rope_frequencies(2, scaling="base", factor=8.0)[0] == [1.0]
    g, m = rows.rope_frequencies(128, scaling="parts", factor=16.0, trained=4096)
    assert math.isclose(m, 0.1 * math.log(16.0) + 1.0) and g[0] == f[0] and math.isclose(g[63], f[63] / 16.0, rel_tol=1e-15)
    turns = [4096 * x / (2 * math.pi) for x in f]
    for a, b, t in zip(f, g, turns):
        assert b == a if t >= 32 else math.isclose(b, a / 16, rel_tol=1e-14) if t <= 1 else a / 16 < b < a
    for kw in (dict(dims=3), dict(dims=0), dict(dims=4, theta=0.0), dict(dims=4, factor=0.5), dict(dims=4, scaling="x"), dict(dims=4, scaling="parts", fast=1.0)):
        with pytest.raises(ValueError):
            rows.rope_frequencies(**kw)


READELF = "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
def test_no_kernel_spills(tmp_path):
    import yaml

    lib = open(rows.library_path(), "rb").read()
    at = lib.index(b"__CLANG_OFFLOAD_BUNDLE__")
    n, pos = struct.unpack_from("<Q", lib, at + 24)[0], at + 32
    for _ in range(n):  # offset, size, length of the target's name, name
        off, size, length = struct.unpack_from("<QQQ", lib, pos)
        if b"gfx950" in lib[pos + 24:pos + 24 + length]:
            (tmp_path / "code.o").write_bytes(lib[at + off:at + off + size])
        pos += 24 + length
    notes = subprocess.run([READELF, "--notes", str(tmp_path / "code.o")], capture_output=True, text=True, check=True).stdout
    kernels = yaml.safe_load(notes[notes.index("---"):notes.index("\n...")])["amdhsa.kernels"]
    assert any("rotate" in k[".name"] for k in kernels) and any("verify" in k[".name"] for k in kernels)
    for k in kernels:
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, k[".name"]
