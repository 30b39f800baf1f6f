"""Latent attention and the bound on all positions together: raised in every form when lens exceed it, and only then."""
import pytest
import torch

import paper_2609_18063_b200 as edg
from test_gpu_latent import FORMS, ONE, SMALL, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS + [edg.LATENT_AUTO])
@pytest.mark.parametrize("lay,new,lens", [(SMALL, [4, 1], [200, 100]), (SMALL, [1], [1]), (SMALL, [1, 70, 3], [3000, 70, 900]), (ONE, [1] * 300, [i % 50 for i in range(300)])])
def test_the_sum_of_lens_against_its_bound(form, lay, new, lens):
    b = Batch(lay, new, lens, form=form)
    for total, status in ((sum(lens) - 1, -4), (sum(lens), 0), (sum(lens) + 1000, 0), (0, -4)):
        b.bounds = b.bounds[:3] + (total,)
        b.ws = torch.zeros(edg.latent_workspace_bytes(b.desc, *b.bounds), dtype=torch.uint8, device="cuda")
        b.y.fill_(7.0)
        b.attend()
        torch.cuda.synchronize()
        assert edg.workspace_status(b.ws) == status
        if status == 0:
            b.check()
