"""Latent attention over and over: the first call against 64 bits, a thousand behind it with the first one's bits."""
import pytest
import torch

import paper_2609_18063_b200 as edg
from test_gpu_latent import LARGE, SMALL, Batch

pytestmark = pytest.mark.gpu


def _again(b, times=1000):
    b.attend()
    b.check()
    first, other = b.y.clone(), torch.zeros((), dtype=torch.bool, device="cuda")
    for _ in range(times):
        b.y.fill_(7.0)
        b.attend()
        other |= (b.y != first).any()
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == 0 and not bool(other)


@pytest.mark.parametrize("new", [[1 + 37 * i % 128 for i in range(150)], [129 + 31 * i % 300 for i in range(60)]])
def test_the_two_threads_of_a_row_exchange_maxima_and_then_sums(new):
    """Prompts of one tile of positions (its maxima are followed by the sums, not by another tile) and of a few, many to a CTA."""
    _again(Batch(SMALL, new, new, form=edg.LATENT_EXPANDED))


def test_the_two_threads_of_a_row_where_cached_positions_lie_before_the_prompt():
    _again(Batch(LARGE, [100] * 40, [100 + 61 * i for i in range(40)], form=edg.LATENT_EXPANDED, page=128))


@pytest.mark.parametrize("form", [edg.LATENT_ABSORBED, edg.LATENT_EXPANDED])
@pytest.mark.parametrize("heads,new,lens", [(8, [1], [1]), (24, [1, 1], [70, 5]), (8, [9, 1], [64, 130]), (8, [3] * 150, [3 + i % 140 for i in range(150)])])
def test_blocks_that_end_with_their_first_tiles(form, heads, new, lens):
    """A block waits for all arrivals of its products before it ends: launches of a tile or two in a row, none behind the other's barriers."""
    _again(Batch(dict(SMALL, heads=heads), new, lens, form=form, page=16))
