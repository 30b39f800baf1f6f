"""Latent attention where the form is left open: batches whose sequences take different forms in one call, and calls that follow one another.

Tolerances are those of the forms by themselves (see test_gpu_latent)."""
import pytest
import torch

import paper_2609_18063_b200 as edg
from test_gpu_latent import LARGE, ODD, ONE, SMALL, WIDE, Batch

pytestmark = pytest.mark.gpu

# long sequences of few new rows beside prompts (two forms in one call), short ones beside prompts (one form)
MIXED = [([300, 1, 40, 0, 3], [300, 4000, 700, 50, 900]), ([1, 65, 64], [5000, 65, 64]), ([2, 129, 1, 257], [1, 4129, 0, 300])]
SHORT = [([300, 1, 40, 0], [300, 90, 70, 5]), ([65], [65]), ([70], [20]), ([1, 100], [1, 100]), ([200, 1], [100, 0])]


@pytest.mark.parametrize("lay", [SMALL, LARGE, ODD, ONE, WIDE])
@pytest.mark.parametrize("new,lens", MIXED + SHORT)
@pytest.mark.parametrize("page", [16, 128])
def test_forms_side_by_side(lay, new, lens, page):
    b = Batch(lay, new, lens, page=page, behind=3)
    b.attend()
    b.check()


def test_forms_by_bounds_that_are_not_met():
    """A caller that captures a call gives bounds above what it has: the same outputs, whichever form they lead to."""
    b = Batch(SMALL, [1, 30, 66], [100, 300, 66])
    b.attend()
    b.check()
    for max_new, total in ((66, 466), (99, 466), (99, 400000)):
        b.bounds = (3, b.T, min(max_new, b.T), total)
        b.ws = torch.zeros(edg.latent_workspace_bytes(b.desc, *b.bounds), dtype=torch.uint8, device="cuda")
        b.y.fill_(7.0)
        b.attend()
        b.check()


@pytest.mark.parametrize("new,lens", [MIXED[0], SHORT[0]])
def test_captured_and_back_to_back(new, lens):
    """Two calls that share a workspace, over and over, in a graph and without."""
    a, b = Batch(SMALL, new, lens), Batch(SMALL, [1] * 4, [700, 3, 64, 2000], seed=1)
    ws = torch.zeros(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device="cuda")
    for _ in range(20):
        a.attend(ws=ws)
        b.attend(ws=ws)
    a.check()
    b.check()
    assert edg.workspace_status(ws) == 0
    first = a.y.clone(), b.y.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):
            a.attend(ws=ws)
            b.attend(ws=ws)
    a.y.fill_(7.0)
    b.y.fill_(7.0)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.y, first[0]) and torch.equal(b.y, first[1]) and edg.workspace_status(ws) == 0


def test_two_calls_at_once():
    """Two streams, each with its own workspace."""
    a, b = Batch(SMALL, *MIXED[0]), Batch(LARGE, [260, 1], [400, 5000], seed=1)
    a.attend()
    b.attend()
    torch.cuda.synchronize()
    first = a.y.clone(), b.y.clone()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        for s, x in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                x.attend()
    torch.cuda.synchronize()
    assert torch.equal(a.y, first[0]) and torch.equal(b.y, first[1])
    a.check()
    b.check()
