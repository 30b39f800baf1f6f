"""Pools from tensors of another type than int32: refused, not read as int32."""
import numpy as np
import pytest
import torch


@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("dtype", ["int64", "int16", "uint8", "float32"])
def test_pools_of_other_types_are_refused(which, dtype):
    from paper_2609_18063_b200 import build
    build.build()
    import paper_2609_18063_b200 as edg
    shapes = ((7,), (3, 4), (3,))
    for make, wide in ((lambda s, d: torch.zeros(s, dtype=getattr(torch, d)), dtype), (lambda s, d: np.zeros(s, dtype=d), dtype)):
        good = [make(s, "int32") for s in shapes]
        assert edg.make_page_pool(*good, page=16).max_pages == 4
        bad = list(good)
        bad[which] = make(shapes[which], wide)
        with pytest.raises(ValueError):
            edg.make_page_pool(*bad, page=16)
