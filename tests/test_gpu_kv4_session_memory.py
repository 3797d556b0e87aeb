"""Memory of the handle that gives places to the rows of a session over the 4-bit cache."""
from __future__ import annotations

import pytest

from paper_2502_11517_amd import kv8
from paper_2502_11517_amd.kv8_session import Session
from test_gpu_kv4_session import SIZES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_rows", [64, 256, 2048])
def test_the_handle_of_places_takes_no_more_memory_than_its_checks_ask_for(max_rows):
    """Its plan and attention are not called: half of what those of the cache would take, at most."""
    s = Session(codes="e2m1", **{**SIZES, "n_q_heads": 32, "n_kv_heads": 8, "head_dim": 128, "max_rows": max_rows})
    as_large = kv8.query_workspace_bytes(kv8.make_config("e4m3", "bf16", 32, 8, 128, 1.0, max_requests=2, max_rows=max_rows, n_phys_pages=60, pages_per_request=30))
    assert s.places_workspace.numel() <= as_large // 2 + (1 << 19)
