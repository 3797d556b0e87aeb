"""The 8-bit cache's library on the CPU: exported symbols, refusals of arguments, sizes.  No call here reaches a launch."""
from __future__ import annotations

import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

import kv8_ref as ref
from paper_2502_11517_amd import kv8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # an aligned address that is never read


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(kv8.library_path()):
        kv8.build_library()


GOOD = dict(codes="e4m3", dtype="bf16", n_q_heads=32, n_kv_heads=8, head_dim=128, softmax_scale=1.0, n_layers=2, max_requests=4, max_rows=64, page_tokens=16,
            n_phys_pages=100, pages_per_request=20)


def config(**kw):
    return kv8.make_config(**{**GOOD, **kw})


def handle(**kw):
    cfg = config(**kw)
    return kv8.PastaKv8(cfg, FAKE, workspace_bytes=kv8.query_workspace_bytes(cfg), page_table=FAKE, k_codes=FAKE, v_codes=FAKE, k_scale=FAKE,
                        v_scale=FAKE, free_pages=FAKE, slot_tag=FAKE, slot_position=FAKE)


def refused(call, code):
    assert call() == code


def test_every_declared_symbol_is_exported():
    hdr = open(os.path.join(ROOT, "include", "pasta_kv8.h")).read()
    declared = set(re.findall(r"\bint32_t\s+(pasta_kv8_\w+)\s*\(", hdr))
    assert declared == {"pasta_kv8_" + n for n in ("create", "destroy", "slots", "append", "plan", "attend")}
    syms = subprocess.run(["nm", "-D", "--defined-only", kv8.library_path()], capture_output=True, text=True).stdout
    assert declared <= {l.split()[-1] for l in syms.splitlines() if " T " in l}


@pytest.mark.parametrize("kw", [dict(codes=2), dict(codes=-1), dict(dtype="f32"), dict(dtype=7), dict(n_q_heads=24), dict(n_q_heads=33), dict(n_q_heads=0),
                                dict(n_kv_heads=0), dict(n_kv_heads=-8), dict(n_q_heads=257, n_kv_heads=257), dict(head_dim=96), dict(head_dim=256),
                                dict(n_layers=0), dict(max_requests=0), dict(max_rows=0), dict(page_tokens=8), dict(page_tokens=24),
                                dict(page_tokens=8192), dict(n_phys_pages=0), dict(pages_per_request=0), dict(softmax_scale=float("nan")),
                                dict(softmax_scale=float("inf")), dict(n_phys_pages=1 << 27), dict(n_phys_pages=1 << 28, page_tokens=4096), dict(pages_per_request=(1 << 23) + 1),
                                dict(pages_per_request=1 << 27), dict(max_requests=1 << 20, pages_per_request=1 << 12), dict(max_rows=1 << 24)])
def test_configurations_that_are_refused(kw):
    with pytest.raises(kv8.PastaError) as e:
        kv8.query_workspace_bytes(config(**kw))
    assert e.value.code == kv8.E_INVAL


def test_struct_sizes_and_addresses():
    cfg = config()
    cfg.struct_size -= 4
    with pytest.raises(kv8.PastaError):
        kv8.query_workspace_bytes(cfg)
    size = kv8.query_workspace_bytes(config())
    for kw, code in ((dict(workspace=FAKE + 16, workspace_bytes=size), kv8.E_INVAL), (dict(workspace=FAKE, workspace_bytes=size - 1), kv8.E_CAPACITY),
                     (dict(workspace=FAKE, workspace_bytes=size, k_codes=FAKE + 8), kv8.E_INVAL),
                     (dict(workspace=FAKE, workspace_bytes=size, slot_tag=FAKE + 1), kv8.E_INVAL),
                     (dict(workspace=FAKE, workspace_bytes=size, v_scale=FAKE + 2), kv8.E_INVAL)):
        with pytest.raises(kv8.PastaError) as e:
            kv8.PastaKv8(config(), **kw)
        assert e.value.code == code


def test_the_workspace_grows_with_rows_and_requests_alone():
    size = kv8.query_workspace_bytes(config())
    assert kv8.query_workspace_bytes(config(n_layers=60, n_phys_pages=1 << 20)) == size
    assert kv8.query_workspace_bytes(config(max_rows=8192)) > size


def test_slots_refusals():
    h = handle()
    good = dict(length=FAKE, row_offsets=FAKE, n_rows=8, slot=FAKE, length_out=FAKE, free_count=FAKE, free_out=FAKE, n_requests=2)
    for kw, code in ((dict(n_requests=5), kv8.E_CAPACITY), (dict(n_rows=65), kv8.E_CAPACITY), (dict(n_requests=-1), kv8.E_INVAL), (dict(n_rows=-1), kv8.E_INVAL),
                     (dict(length=None), kv8.E_INVAL), (dict(row_offsets=None), kv8.E_INVAL), (dict(slot=None), kv8.E_INVAL),
                     (dict(length_out=None), kv8.E_INVAL), (dict(free_count=None), kv8.E_INVAL), (dict(free_out=None), kv8.E_INVAL),
                     (dict(keep=FAKE + 2), kv8.E_INVAL), (dict(row_position=FAKE + 1), kv8.E_INVAL)):
        refused(h.prepare_slots(**{**good, **kw}), code)
    cfg = config()
    for left_out in ("page_table", "free_pages", "slot_tag", "slot_position"):
        bufs = {k: FAKE for k in ("page_table", "free_pages", "slot_tag", "slot_position") if k != left_out}
        h = kv8.PastaKv8(cfg, FAKE, workspace_bytes=1 << 40, **bufs)
        refused(h.prepare_slots(**good, row_tag=FAKE, row_position=FAKE), kv8.E_INVAL)


def test_append_refusals():
    h = handle()
    good = dict(layer=0, slot=FAKE, k_new=FAKE, v_new=FAKE, n_rows=4, dtype="bf16")
    for kw, code in ((dict(layer=2), kv8.E_INVAL), (dict(layer=-1), kv8.E_INVAL), (dict(n_rows=-1), kv8.E_INVAL), (dict(n_rows=65), kv8.E_CAPACITY),
                     (dict(dtype=3), kv8.E_INVAL), (dict(slot=None), kv8.E_INVAL), (dict(k_new=None), kv8.E_INVAL), (dict(v_new=None), kv8.E_INVAL),
                     (dict(k_new=FAKE + 8), kv8.E_INVAL), (dict(slot=FAKE + 1), kv8.E_INVAL), (dict(n_rows=0, slot=None), kv8.OK)):
        refused(h.prepare_append(**{**good, **kw}), code)
    h = kv8.PastaKv8(config(), FAKE, workspace_bytes=1 << 40, k_codes=FAKE, v_codes=FAKE, k_scale=FAKE)
    refused(h.prepare_append(**good), kv8.E_INVAL)


def test_plan_and_attend_refusals():
    h = handle()
    plan = dict(length=FAKE, row_offsets=FAKE, n_rows=8, n_requests=2)
    for kw, code in ((dict(n_requests=5), kv8.E_CAPACITY), (dict(n_rows=65), kv8.E_CAPACITY), (dict(n_rows=-1, max_request_rows=1), kv8.E_INVAL),
                     (dict(max_request_rows=-1), kv8.E_INVAL), (dict(length=None), kv8.E_INVAL), (dict(row_offsets=None), kv8.E_INVAL),
                     (dict(prefix_len=FAKE + 1), kv8.E_INVAL)):
        refused(h.prepare_plan(**{**plan, **kw}), code)
    good = dict(layer=0, q=FAKE, out=FAKE, n_rows=8)
    refused(h.prepare_attend(**good), kv8.E_STATE)  # no plan yet
    refused(h.prepare_plan(**{**plan, "n_rows": 0}), kv8.OK)  # (no launch)
    refused(h.prepare_attend(**good), kv8.E_STATE)  # a plan of other rows
    for kw, code in ((dict(layer=2), kv8.E_INVAL), (dict(layer=-1), kv8.E_INVAL), (dict(logit_cap=-1.0), kv8.E_INVAL), (dict(logit_cap=float("nan")), kv8.E_INVAL),
                     (dict(logit_cap=float("inf")), kv8.E_INVAL), (dict(row_position=FAKE), kv8.E_INVAL), (dict(n_rows=0, q=None, out=None), kv8.OK)):
        refused(h.prepare_attend(**{**good, "n_rows": 0, **kw}), code)


def test_destroyed_handles_and_wrong_structs():
    h = handle()
    lib = kv8.load_library()
    a = kv8.PlanArgs(4)
    assert lib.pasta_kv8_plan(h._h, C.byref(a)) == kv8.E_INVAL
    a = kv8.AttendArgs(C.sizeof(kv8.AttendArgs), 1)
    assert lib.pasta_kv8_attend(h._h, C.byref(a)) == kv8.E_INVAL  # unknown flags
    assert lib.pasta_kv8_attend(None, C.byref(a)) == kv8.E_STATE
    assert lib.pasta_kv8_destroy(None) == kv8.OK


def test_tensors_are_checked_for_type_contiguity_and_size():
    import torch

    h = handle()
    i32 = torch.zeros(8, dtype=torch.int32)
    with pytest.raises(ValueError):
        h.prepare_plan(i32.long()[:2], i32, 8)
    with pytest.raises(ValueError):
        h.prepare_plan(i32[:2], torch.zeros(16, dtype=torch.int32)[::2], 8)
    with pytest.raises(ValueError):
        h.prepare_plan(i32[:2], i32[:2], 8)
    with pytest.raises(ValueError):
        h.prepare_attend(0, torch.zeros(8, 32, 128), torch.zeros(8, 32, 128, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        h.prepare_append(0, i32, torch.zeros(8, 8, 128, dtype=torch.bfloat16), torch.zeros(8, 8, 128))
    with pytest.raises(ValueError):
        h.prepare_append(0, i32, torch.zeros(8, 128, 8).transpose(1, 2), torch.zeros(8, 8, 128))
    with pytest.raises(ValueError):
        kv8.PastaKv8(config(), torch.empty(1 << 20, dtype=torch.uint8), page_table=torch.zeros(3, 20, dtype=torch.int32))


def test_the_reference_codes_are_torchs():
    import torch

    b = torch.arange(256, dtype=torch.uint8)
    v = b.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, ref.code_values("e4m3"), equal_nan=True)
    x = np.random.default_rng(0).standard_normal(5000) * 100
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(ref.nearest(x.astype(np.float64), "e4m3"), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


READELF = "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
def test_no_kernel_spills(tmp_path):
    """What the compiler gave the kernels: no scratch memory, no spilled vector registers, two work-groups of the attention per CU."""
    import struct

    import yaml

    lib = open(kv8.library_path(), "rb").read()
    at = lib.index(b"__CLANG_OFFLOAD_BUNDLE__")
    n, pos = struct.unpack_from("<Q", lib, at + 24)[0], at + 32
    for _ in range(n):  # offset, size, length of the target's name, name
        off, size, length = struct.unpack_from("<QQQ", lib, pos)
        if b"gfx950" in lib[pos + 24:pos + 24 + length]:
            (tmp_path / "code.o").write_bytes(lib[at + off:at + off + size])
        pos += 24 + length
    notes = subprocess.run([READELF, "--notes", str(tmp_path / "code.o")], capture_output=True, text=True, check=True).stdout
    kernels = yaml.safe_load(notes[notes.index("---"):notes.index("\n...")])["amdhsa.kernels"]
    attend = [k for k in kernels if "k8_attend" in k[".name"]]
    assert len(attend) == 24
    for k in kernels:
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, k[".name"]
    for k in attend:
        assert k[".vgpr_count"] <= 256 and 2 * k[".group_segment_fixed_size"] <= 160 * 1024, k[".name"]
