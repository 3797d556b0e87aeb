"""A host tensor where the kernels want device memory is refused ahead of any launch, whichever argument it is."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2502_11517_amd import kv8

FAKE = 0x10000  # an aligned address that is never read
BUFFERS = dict(page_table=(torch.int32, (4, 20)), k_codes=(torch.uint8, (2, 100, 8, 1, 8, 16, 16)), v_codes=(torch.uint8, (2, 100, 8, 1, 128, 16)),
               k_scale=(torch.float32, (2, 100, 8, 1)), v_scale=(torch.float32, (2, 100, 8, 1)), free_pages=(torch.int32, (100,)),
               slot_tag=(torch.uint8, (1600,)), slot_position=(torch.int32, (1600,)))


def config():
    return kv8.make_config("e4m3", "bf16", 32, 8, 128, 1.0, n_layers=2, max_requests=4, max_rows=64, n_phys_pages=100, pages_per_request=20)


def handle(**kw):
    return kv8.PastaKv8(config(), **{**dict(workspace=FAKE, workspace_bytes=1 << 40), **{k: FAKE for k in BUFFERS}, **kw})


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(kv8.library_path()):
        kv8.build_library()


@pytest.mark.parametrize("name", [*BUFFERS, "workspace"])
def test_a_handles_buffers(name):
    if name == "workspace":
        bad = torch.zeros(kv8.query_workspace_bytes(config()) + 256, dtype=torch.uint8)
        bad = bad[-bad.data_ptr() % 256:]
    else:
        dtype, shape = BUFFERS[name]
        bad = torch.zeros(shape, dtype=dtype)
    with pytest.raises(ValueError, match="device memory"):
        handle(**{name: bad})


I32, U8, F32 = torch.int32, torch.uint8, torch.float32
CALLS = {
    "slots": (dict(n_requests=2, n_rows=8, length=FAKE, row_offsets=FAKE, slot=FAKE, length_out=FAKE, free_count=FAKE, free_out=FAKE),
              dict(length=I32, row_offsets=I32, slot=I32, length_out=I32, free_count=I32, free_out=I32, keep=I32, row_tag=U8, row_position=I32)),
    "append": (dict(layer=0, n_rows=8, slot=FAKE, k_new=FAKE, v_new=FAKE, dtype="bf16"), dict(slot=I32, k_new=torch.bfloat16, v_new=torch.bfloat16)),
    "plan": (dict(n_requests=2, n_rows=8, length=FAKE, row_offsets=FAKE), dict(length=I32, row_offsets=I32, prefix_len=I32, slot=I32)),
    "attend": (dict(layer=0, n_rows=8, q=FAKE, out=FAKE), dict(q=torch.bfloat16, out=torch.bfloat16, lse=F32, slopes=F32, row_see=torch.int64, row_position=I32)),
}


@pytest.mark.parametrize("call,name", [(c, n) for c, (_, names) in CALLS.items() for n in names])
def test_a_calls_arguments(call, name):
    good, types = CALLS[call]
    h = handle()
    getattr(h, "prepare_" + call)(**good)
    with pytest.raises(ValueError, match=name + ".*device memory"):
        getattr(h, "prepare_" + call)(**{**good, name: torch.zeros(8 * 32 * 128, dtype=types[name])})


@pytest.mark.parametrize("call", CALLS)
def test_a_prepared_call_of_a_destroyed_handle_does_not_reach_its_memory(call, monkeypatch):
    h = handle()
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda handle, args: seen.append(handle) or kv8.E_STATE

    monkeypatch.setattr(h, "_lib", Library())
    prepared = getattr(h, "prepare_" + call)(**CALLS[call][0])
    h._h = None  # what destroy() leaves
    assert prepared() == kv8.E_STATE and seen == [None]
    monkeypatch.undo()
    h = handle()
    prepared = getattr(h, "prepare_" + call)(**CALLS[call][0])
    h.destroy()
    assert prepared() == kv8.E_STATE
