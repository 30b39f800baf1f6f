"""Latent attention and row bounds that contradict one another: reported, done in bounded time, nothing written outside."""
import pytest
import torch

import paper_2609_18063_b200 as edg
from test_gpu_latent import FORMS, SMALL, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS + [edg.LATENT_AUTO])
def test_sequences_that_overlap_are_reported(form):
    """cu that goes back and forth: half of 400 sequences claim all rows."""
    n, T = 400, 300
    b = Batch(SMALL, [T] + [0] * (n - 1), [700] * n, form=form)
    b.bounds = (n, T, T, 700 * n)
    b.ws = torch.zeros(edg.latent_workspace_bytes(b.desc, *b.bounds), dtype=torch.uint8, device="cuda")
    guard = torch.full((T + 64, SMALL["heads"], SMALL["dv"]), 7.0, dtype=b.y.dtype, device="cuda")
    b.y = guard[32:32 + T]
    b.cu = torch.tensor([0, T] * (n // 2) + [0], dtype=torch.int32, device="cuda")
    b.attend()
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == -4
    assert (guard[:32] == 7.0).all() and (guard[32 + T:] == 7.0).all()
    b.cu.copy_(torch.tensor([0] + [T] * n, dtype=torch.int32))      # the same call, with rows that hold: the workspace is none the worse
    b.ws.zero_()
    b.attend()
    b.check()
