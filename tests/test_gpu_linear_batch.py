"""The int4 projection: what a token gets does not depend on the other tokens of its call."""
import pytest
import torch

from test_gpu_linear import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,rank,out", [(577, 16, "f32"), (6144, 0, "bf16"), (40001, 0, "f32")])
@pytest.mark.parametrize("T", [2, 8, 9, 16, 40, 64])
def test_a_token_keeps_its_bits_whatever_stands_beside_it(N, rank, out, T):
    """With T fixed: others, far larger and smaller ones, zeros, infinities and NaN in all rows but three."""
    c = Case(N, 2048, 64, rank, T, out)
    c.run()
    c.check()
    first, kept = c.y.clone(), sorted({0, T // 2, T - 1})
    mask = torch.zeros((T, 1), dtype=torch.bool, device="cuda")
    mask[kept] = True
    x0 = c.dev[0].clone()
    for k, scale in enumerate((1.0, 1e20, 1e-20, 0.0, float("inf"), float("nan"))):
        other = torch.randn(x0.shape, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda") * scale
        c.dev[0].copy_(torch.where(mask, x0, other.bfloat16()))
        c.y.fill_(7.0)
        c.run()
        assert torch.equal(c.y[kept], first[kept])
