"""The 4-bit cache's library on the CPU: exported symbols, refusals of arguments, sizes, what the compiler gave the kernels.  No call here reaches a launch."""
from __future__ import annotations

import ctypes as C
import os
import re
import struct
import subprocess

import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2502_11517_amd import kv4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # an aligned address that is never read


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(kv4.library_path()):
        kv4.build_library()


GOOD = dict(dtype="bf16", n_q_heads=32, n_kv_heads=8, head_dim=128, softmax_scale=1.0, n_layers=2, max_requests=4, max_rows=64, page_tokens=16,
            n_phys_pages=100, pages_per_request=20)
BUFS = dict(page_table=FAKE, k_codes=FAKE, v_codes=FAKE, k_scale=FAKE, v_scale=FAKE, slot_tag=FAKE, slot_position=FAKE)


def config(**kw):
    return kv4.make_config(**{**GOOD, **kw})


def handle(left_out=(), **kw):
    cfg = config(**kw)
    return kv4.PastaKv4(cfg, FAKE, workspace_bytes=kv4.query_workspace_bytes(cfg), **{k: v for k, v in BUFS.items() if k not in left_out})


def test_every_declared_symbol_is_exported():
    hdr = open(os.path.join(ROOT, "include", "pasta_kv4.h")).read()
    declared = set(re.findall(r"\bint32_t\s+(pasta_kv4_\w+)\s*\(", hdr))
    assert declared == {"pasta_kv4_" + n for n in ("create", "destroy", "append", "read", "plan", "attend")}
    syms = subprocess.run(["nm", "-D", "--defined-only", kv4.library_path()], capture_output=True, text=True).stdout
    assert declared <= {l.split()[-1] for l in syms.splitlines() if " T " in l}


@pytest.mark.parametrize("kw", [dict(dtype="f32"), dict(dtype=7), dict(n_q_heads=24), dict(n_q_heads=33), dict(n_q_heads=0), dict(n_kv_heads=0),
                                dict(n_kv_heads=-8), dict(n_q_heads=257, n_kv_heads=257), dict(head_dim=96), dict(head_dim=256), dict(n_layers=0),
                                dict(max_requests=0), dict(max_rows=0), dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=8192),
                                dict(n_phys_pages=0), dict(pages_per_request=0), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")),
                                dict(n_phys_pages=1 << 27), dict(n_phys_pages=1 << 28, page_tokens=4096), dict(pages_per_request=(1 << 23) + 1),
                                dict(max_requests=1 << 20, pages_per_request=1 << 12), dict(max_rows=1 << 24)])
def test_configurations_that_are_refused(kw):
    with pytest.raises(kv4.PastaError) as e:
        kv4.query_workspace_bytes(config(**kw))
    assert e.value.code == kv4.E_INVAL


def test_struct_sizes_and_addresses():
    cfg = config()
    cfg.struct_size -= 4
    with pytest.raises(kv4.PastaError):
        kv4.query_workspace_bytes(cfg)
    size = kv4.query_workspace_bytes(config())
    for kw, code in ((dict(workspace=FAKE + 16, workspace_bytes=size), kv4.E_INVAL), (dict(workspace=FAKE, workspace_bytes=size - 1), kv4.E_CAPACITY),
                     (dict(k_codes=FAKE + 8), kv4.E_INVAL), (dict(v_scale=FAKE + 4), kv4.E_INVAL), (dict(slot_tag=FAKE + 1), kv4.E_INVAL),
                     (dict(page_table=FAKE + 2), kv4.E_INVAL)):
        with pytest.raises(kv4.PastaError) as e:
            kv4.PastaKv4(config(), **kw)
        assert e.value.code == code


def test_append_refusals():
    h = handle()
    good = dict(layer=0, slot=FAKE, k_new=FAKE, v_new=FAKE, n_rows=4, dtype="bf16")
    for kw, code in ((dict(layer=2), kv4.E_INVAL), (dict(layer=-1), kv4.E_INVAL), (dict(n_rows=-1), kv4.E_INVAL), (dict(n_rows=65), kv4.E_CAPACITY),
                     (dict(dtype=3), kv4.E_INVAL), (dict(slot=None), kv4.E_INVAL), (dict(k_new=None), kv4.E_INVAL), (dict(v_new=None), kv4.E_INVAL),
                     (dict(k_new=FAKE + 8), kv4.E_INVAL), (dict(slot=FAKE + 1), kv4.E_INVAL), (dict(n_rows=0, slot=None), kv4.OK)):
        assert h.prepare_append(**{**good, **kw})() == code, kw
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        assert handle(left_out=[name]).prepare_append(**good)() == kv4.E_INVAL


def test_read_refusals():
    h = handle()
    good = dict(layer=1, slot=FAKE, k_out=FAKE, v_out=FAKE, n_rows=400, dtype="f32")
    for kw, code in ((dict(layer=2), kv4.E_INVAL), (dict(layer=-1), kv4.E_INVAL), (dict(n_rows=-1), kv4.E_INVAL), (dict(dtype=5), kv4.E_INVAL),
                     (dict(n_rows=(1 << 27) + 1), kv4.E_CAPACITY), (dict(slot=None), kv4.E_INVAL), (dict(k_out=None, v_out=None), kv4.E_INVAL), (dict(v_out=FAKE + 4), kv4.E_INVAL),
                     (dict(n_rows=0, slot=None, k_out=None, v_out=None), kv4.OK)):
        assert h.prepare_read(**{**good, **kw})() == code, kw
    assert handle(left_out=["v_scale"]).prepare_read(**good)() == kv4.E_INVAL
    assert handle(left_out=["k_codes"]).prepare_read(**good)() == kv4.E_INVAL


@pytest.mark.parametrize("stride,code", [(8 * 128 - 8, kv4.E_INVAL), (8 * 128 + 4, kv4.E_INVAL), (-1024, kv4.E_INVAL), (1 << 50, kv4.E_INVAL)])
def test_strides_that_are_refused(stride, code):
    h = handle()
    lib = kv4.load_library()
    for fields in ((stride, 0), (0, stride)):
        a = kv4.AppendArgs(C.sizeof(kv4.AppendArgs), 0, 0, 4, kv4.BF16, FAKE, FAKE, FAKE, *fields)
        assert lib.pasta_kv4_append(h._h, C.byref(a)) == code
        a = kv4.ReadArgs(C.sizeof(kv4.ReadArgs), 0, 0, 4, kv4.BF16, FAKE, FAKE, FAKE, *fields)
        assert lib.pasta_kv4_read(h._h, C.byref(a)) == code


def test_plan_and_attend_refusals():
    h = handle()
    plan = dict(length=FAKE, row_offsets=FAKE, n_rows=8, n_requests=2)
    for kw, code in ((dict(n_requests=5), kv4.E_CAPACITY), (dict(n_rows=65), kv4.E_CAPACITY), (dict(n_rows=-1, max_request_rows=1), kv4.E_INVAL),
                     (dict(max_request_rows=-1), kv4.E_INVAL), (dict(length=None), kv4.E_INVAL), (dict(row_offsets=None), kv4.E_INVAL),
                     (dict(prefix_len=FAKE + 1), kv4.E_INVAL)):
        assert h.prepare_plan(**{**plan, **kw})() == code, kw
    good = dict(layer=0, q=FAKE, out=FAKE, n_rows=8)
    assert h.prepare_attend(**good)() == kv4.E_STATE  # no plan yet
    assert h.prepare_plan(**{**plan, "n_rows": 0})() == kv4.OK  # (no launch)
    assert h.prepare_attend(**good)() == kv4.E_STATE  # a plan of other rows
    for kw, code in ((dict(layer=2), kv4.E_INVAL), (dict(layer=-1), kv4.E_INVAL), (dict(logit_cap=-1.0), kv4.E_INVAL),
                     (dict(logit_cap=float("nan")), kv4.E_INVAL), (dict(logit_cap=float("inf")), kv4.E_INVAL), (dict(row_position=FAKE), kv4.E_INVAL),
                     (dict(n_rows=0, q=None, out=None), kv4.OK)):
        assert h.prepare_attend(**{**good, "n_rows": 0, **kw})() == code, kw
    for name in ("page_table", "k_codes", "v_scale"):
        h = handle(left_out=[name])
        assert h.prepare_plan(**{**plan, "n_rows": 0})() == (kv4.E_INVAL if name == "page_table" else kv4.OK)
        assert h.prepare_attend(**{**good, "n_rows": 0})() in (kv4.E_INVAL, kv4.E_STATE)


def test_destroyed_handles_and_wrong_structs():
    h = handle()
    lib = kv4.load_library()
    for name, args in (("append", kv4.AppendArgs), ("read", kv4.ReadArgs), ("plan", kv4.PlanArgs), ("attend", kv4.AttendArgs)):
        f = getattr(lib, "pasta_kv4_" + name)
        assert f(h._h, C.byref(args(4))) == kv4.E_INVAL and f(h._h, C.byref(args(C.sizeof(args), 1))) == kv4.E_INVAL
        assert f(None, C.byref(args(C.sizeof(args)))) == kv4.E_STATE and f(h._h, None) == kv4.E_INVAL
    call = h.prepare_append(0, FAKE, FAKE, FAKE, n_rows=4, dtype="bf16")
    h.destroy()
    assert call() == kv4.E_STATE and lib.pasta_kv4_destroy(None) == kv4.OK


def test_tensors_are_checked():
    h = handle()
    i32 = torch.zeros(8, dtype=torch.int32)
    bf = torch.zeros(8, 8, 128, dtype=torch.bfloat16)
    for k, v in ((bf, torch.zeros(8, 8, 128)), (bf.transpose(0, 1), bf), (bf[:, :, ::2], bf), (bf[:4], bf), (bf[:1].expand(8, 8, 128), bf),
                 (torch.zeros(8, 128, 8, dtype=torch.bfloat16).transpose(1, 2), bf), (bf, bf)):
        with pytest.raises(ValueError):  # (the last one: host memory)
            h.prepare_append(0, FAKE, k, v, n_rows=8)
        with pytest.raises(ValueError):
            h.prepare_read(0, FAKE, k, v, n_rows=8)
    with pytest.raises(ValueError):
        h.prepare_plan(i32.long()[:2], i32, 8)
    with pytest.raises(ValueError):
        kv4.PastaKv4(config(), page_table=torch.zeros(3, 20, dtype=torch.int32))


def test_the_reference_packs_what_it_unpacks():
    rng = np.random.default_rng(0)
    cfg = config(n_layers=1, n_phys_pages=3, page_tokens=32, n_kv_heads=2, n_q_heads=2)
    bufs = [rng.integers(0, 256, s).astype(np.uint8) for s in kv4.cache_shapes(cfg)]
    c = ref.Cache.unpack(3, 2, 32, 128, *(b[0] for b in bufs))
    for got, want in zip(c.pack(), bufs):
        assert np.array_equal(got.reshape(want.shape[1:]), want[0])
    # a value where include/pasta_kv4.h says: page 2, head 1, token 21 of it, dim 77
    assert c.kc[2, 1, 21, 77] == bufs[0][0, 2, 1, 1, 77 // 32, 5, 77 % 32 // 2] >> 4 * (77 & 1) & 15
    assert c.vc[2, 1, 21, 77] == bufs[1][0, 2, 1, 1, 77, 5 // 2] >> 4 * (5 & 1) & 15


READELF = "/opt/rocm/llvm/bin/llvm-readelf"


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
def test_no_kernel_spills(tmp_path):
    """No scratch memory, no spilled vector registers (but for one kernel, in a way that is rare), two work-groups of the attention per CU."""
    import yaml

    lib = open(kv4.library_path(), "rb").read()
    at = lib.index(b"__CLANG_OFFLOAD_BUNDLE__")
    n, pos = struct.unpack_from("<Q", lib, at + 24)[0], at + 32
    for _ in range(n):  # offset, size, length of the target's name, name
        off, size, length = struct.unpack_from("<QQQ", lib, pos)
        if b"gfx950" in lib[pos + 24:pos + 24 + length]:
            (tmp_path / "code.o").write_bytes(lib[at + off:at + off + size])
        pos += 24 + length
    notes = subprocess.run([READELF, "--notes", str(tmp_path / "code.o")], capture_output=True, text=True, check=True).stdout
    kernels = yaml.safe_load(notes[notes.index("---"):notes.index("\n...")])["amdhsa.kernels"]
    attend = [k for k in kernels if "k4_attend" in k[".name"]]
    assert attend
    for k in kernels:
        if "k4_attendILi128ELb1ELb1ELi0E" in k[".name"]:  # (two groups of fp16 rows of 128 dims: a few registers, where V's scales are far apart)
            assert k[".private_segment_fixed_size"] <= 24
            continue
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, k[".name"]
    for k in attend:
        assert k[".vgpr_count"] <= 256 and 2 * k[".group_segment_fixed_size"] <= 160 * 1024, k[".name"]
