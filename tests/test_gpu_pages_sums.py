"""Pages asked for beyond what 32 bits count: refused like any list that the pool cannot serve."""
import pytest
import torch

import paper_2609_18063_b200 as edg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,each,short", [(64, 2 ** 26, True), (63, 2 ** 26, True), (64, 2 ** 26 - 1, True), (48, 2 ** 26, True), (1, 2 ** 26, True), (64, 1, False)])
def test_a_list_whose_sum_is_beyond_32_bits(n, each, short):
    """64 sequences of 2^26 pages each: 2^32 in all.  The table of such a pool takes 16 GB."""
    page, most, n_pages = 1, 2 ** 26, 100
    refs, lens = torch.zeros(n_pages, dtype=torch.int32, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    table = torch.full((64, most), -1, dtype=torch.int32, device="cuda")
    rows = torch.zeros((1, n_pages, page, 8), dtype=torch.bfloat16, device="cuda")
    pool, cache = edg.make_page_pool(refs, table, lens, page=page), edg.make_page_cache(rows)
    ws = torch.zeros(edg.pages_workspace_bytes(pool), dtype=torch.uint8, device="cuda")
    seqs, counts = torch.arange(n, dtype=torch.int32, device="cuda"), torch.full((n,), each, dtype=torch.int32, device="cuda")
    edg.pages_reserve(pool, cache, n, seqs, counts, ws)
    torch.cuda.synchronize()
    assert edg.workspace_status(ws) == (-3 if short else 0)
    assert lens.tolist() == ([0] * 64 if short else [each] * n)
    assert int(refs.sum()) == (0 if short else n * each) and int((table[:, :2] >= 0).sum()) == (0 if short else n)
