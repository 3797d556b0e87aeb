"""Heads whose V is 0 throughout (scales of 2^-100, the least there are): out is 0 and lse what the scores say, however many tokens there are."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2502_11517_amd import kv4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("byte", [27, 30, 127, 246])
@pytest.mark.parametrize("requests,rows", [(70, 1), (70, 40), (1, 1), (2, 3)])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64)])
def test_many_tokens_of_equal_scores_behind_some_of_lower_ones(dtype, D, requests, rows, byte):
    """All requests hold the same pages (70: no tile is split; 1 and 2: pieces).  Scores are 0 in the first 4 of every 16 pages of 64 tokens and 7.9 log2 units in
    the others, so that weights are up to 2^15 of their base and sums as large as they get.  lse is off by 2^-20 (1 + |s| + |lse|), as everywhere, and by the
    weights' own sum in fp32: sums of T / 4 terms, 16 at a time, 2^-24 of each of T / 64 partial sums at most, which is T * 2^-30 relative."""
    T, P, H, G = 131072, 64, 8, 1
    pages = T // P
    cfg = kv4.make_config(dtype, H * G, H, D, 1.0, max_requests=requests, max_rows=requests * rows, page_tokens=P, n_phys_pages=pages, pages_per_request=pages)
    u8 = dict(dtype=torch.uint8, device="cuda")
    k, v, ks, vs = (torch.zeros(s, **u8) for s in kv4.cache_shapes(cfg))
    ks.fill_(127), vs.fill_(byte)
    low = torch.arange(pages, device="cuda") % 16 < 4
    k[0, ~low, :, :, 0, :, 0] = 2  # dim 0 is 1
    table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(requests, pages).contiguous()
    n = requests * rows
    td = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    s = 5.46875  # 7.89 log2 units, a bf16 number
    q = torch.zeros(n, H * G, D, dtype=td, device="cuda")
    q[:, :, 0] = s
    out, lse = torch.full_like(q, 7.0), torch.full((n, H * G), 7.0, device="cuda")
    h = kv4.PastaKv4(cfg, torch.empty(kv4.query_workspace_bytes(cfg), **u8), page_table=table, k_codes=k, v_codes=v, k_scale=ks, v_scale=vs,
                     stream=torch.cuda.current_stream().cuda_stream)
    h.plan(torch.full((requests,), T, dtype=torch.int32, device="cuda"), torch.arange(requests + 1, dtype=torch.int32, device="cuda") * rows, n, max_request_rows=rows)
    h.attend(0, q, out, lse=lse)
    torch.cuda.synchronize()
    assert (out == 0).all()
    lse = lse.double().cpu().numpy().reshape(requests, rows, H)
    for i in range(rows):
        t = np.arange(T - rows + 1 + i)
        many = int((t // P % 16 >= 4).sum())
        want = np.log(many * np.exp(s) + len(t) - many)
        assert (np.abs(lse[:, i] - want) <= 2.0 ** -20 * (1 + s + want) + T * 2.0 ** -30).all(), (i, lse[:, i].min(), lse[:, i].max(), want)
