"""Latent attention, expanded form: values and weights are held in 11 bits where their range allows it, and in the range of bf16 where it does not.

What the roundings leave, to first order and as in _latent_ref: keys are bf16 (half a step 2^-8, taken as uniform, which is the most that it leaves in the
mean), values and weights fp16 (2^-11), the output fp16 (2^-11).  In the mean square over a batch this is a bound, not an estimate: a rounding is
at most half a step, and below it for all but the smallest mantissas."""
import math

import pytest
import torch

import paper_2609_18063_b200 as edg
from _latent_ref import attention, context
from test_gpu_latent import LARGE, ODD, SMALL, Batch

pytestmark = pytest.mark.gpu


def _sigma(b):
    """(y, sigma) [T][heads][d_v] with fp16 values, weights and outputs and bf16 keys; NaN behind the last sequence"""
    y, _ = attention(b.cache, b.table, b.cu_host, b.lens_host, b.q, b.q_rope, b.W_uk, b.W_uv, b.scale)
    var = torch.full_like(y, math.nan)
    for i, n in enumerate(b.lens_host):
        r0, r1 = b.cu_host[i], b.cu_host[i + 1]
        m = r1 - r0
        if m == 0:
            continue
        rows = context(b.cache, b.table[i], n)
        c, pos = rows[:, :b.dl], rows[:, b.dl:]
        seen = torch.arange(n, device="cuda")[None] <= (n - m + torch.arange(m, device="cuda"))[:, None]
        for h in range(y.shape[1]):
            key, val = c @ b.W_uk[h].double().T, c @ b.W_uv[h].double().T
            qn, qr = b.q[r0:r1, h, :b.dn].double(), b.q_rope[r0:r1, h].double()
            s = (b.scale * (qn @ key.T + qr @ pos.T)).masked_fill(~seen, -math.inf)
            p2 = torch.softmax(s, dim=1) ** 2
            o = y[r0:r1, h]
            w = p2 * b.scale ** 2 * (qn ** 2 @ (key ** 2).T)
            keys = (w @ val ** 2 - 2 * o * (w @ val) + o ** 2 * w.sum(dim=1, keepdim=True)).clamp(min=0)
            var[r0:r1, h] = (2.0 ** -16 * keys + 2.0 ** -22 * (2 * (p2 @ val ** 2) + o ** 2)) / 3
    return y, var.sqrt()


@pytest.mark.parametrize("lay", [SMALL, LARGE, ODD])
@pytest.mark.parametrize("new,lens", [([500], [500]), ([128, 300, 1, 70], [128, 700, 129, 470])])
def test_values_and_weights_of_prompts_keep_eleven_bits(lay, new, lens):
    b = Batch(lay, new, lens, form=edg.LATENT_EXPANDED, out="f16")
    b.attend()
    b.check()
    y, sigma = _sigma(b)
    off = b.y.double() - y
    assert (off ** 2).mean().sqrt() <= (sigma ** 2).mean().sqrt()


def _columns(b):
    """Every output within its own column's bound: six deviations with all roundings of bf16, half a step of the output, 2^-16 of the column's largest"""
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == 0
    y, sigma = attention(b.cache, b.table, b.cu_host, b.lens_host, b.q, b.q_rope, b.W_uk, b.W_uv, b.scale)
    got = b.y.double()
    tol = 6 * sigma + 2.0 ** -8 * (y.abs() + 6 * sigma) + 2.0 ** -16 * y.abs().amax(dim=0, keepdim=True)
    assert torch.isfinite(got).all() and ((got - y).abs() <= tol).all()


@pytest.mark.parametrize("values", [1e-30, 1e-9, 2.0 ** -13, 2.0 ** -8, 1.0, 2.0 ** 6, 1e4, 1e20])
def test_values_of_any_magnitude(values):
    """What W_uv makes of a row, from far below fp16 to far above it"""
    b = Batch(SMALL, [300, 1], [400, 200], form=edg.LATENT_EXPANDED)
    b.W_uv = (b.W_uv.float() * values).bfloat16()
    b.attend()
    _columns(b)


@pytest.mark.parametrize("small", [1e-30, 1e-6, 2.0 ** -9, 0.0])
def test_columns_of_different_magnitude(small):
    b = Batch(SMALL, [300, 1], [400, 200], form=edg.LATENT_EXPANDED)
    b.W_uv = b.W_uv.clone()
    b.W_uv[:, ::3] = (b.W_uv[:, ::3].float() * small).bfloat16()
    b.attend()
    _columns(b)
    if small == 0.0:
        assert (b.y[:, :, ::3] == 0).all()


@pytest.mark.parametrize("value", [1e30, 1e4, 100.0, 1e-4, 1e-30, 0.0])
@pytest.mark.parametrize("where", [5, 130, 290])
def test_rows_of_another_magnitude_in_a_tile(value, where):
    """One cache row far larger or smaller than those around it, tiles of both kinds in one call; rows before it are compared (behind it a large one may
    take all weight, or scores leave fp32)."""
    b = Batch(SMALL, [400, 30], [400, 90], form=edg.LATENT_EXPANDED)
    at = (int(b.table[0, where // 64]), where % 64)
    b.cache[at][:b.dl] = (torch.sign(b.cache[at][:b.dl].float()) * value).bfloat16()
    b.attend()
    torch.cuda.synchronize()
    y, sigma = attention(b.cache, b.table, b.cu_host, b.lens_host, b.q, b.q_rope, b.W_uk, b.W_uv, b.scale)
    keep = [t for t in range(430) if t < where or t >= 400 or value <= 1.0]
    tol = 6 * sigma + 2.0 ** -8 * (y.abs() + 6 * sigma) + 2.0 ** -16 * y[keep].abs().max()
    assert ((b.y.double() - y).abs() <= tol)[keep].all()


def test_rows_of_zeros_and_values_of_zeros():
    b = Batch(SMALL, [200], [200], form=edg.LATENT_EXPANDED)
    b.cache[:, ::2, :b.dl] = 0
    b.attend()
    b.check()
    b.W_uv = torch.zeros_like(b.W_uv)
    b.attend()
    torch.cuda.synchronize()
    assert (b.y == 0).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), 1e30])
def test_weights_that_are_not_of_this_world_stay_in_their_column(value):
    """A row of W_uv that is not finite, or does not fit, makes its own column so and no other"""
    b = Batch(SMALL, [200, 3], [200, 90], form=edg.LATENT_EXPANDED)
    clean = b.W_uv.clone()
    b.W_uv = clean.clone()
    b.W_uv[3, 7] = value
    b.attend()
    torch.cuda.synchronize()
    y, sigma = attention(b.cache, b.table, b.cu_host, b.lens_host, b.q, b.q_rope, b.W_uk, clean, b.scale)
    tol = 6 * sigma + 2.0 ** -8 * (y.abs() + 6 * sigma) + 2.0 ** -16 * y.abs().max()
    ok = (b.y.double() - y).abs() <= tol
    ok[:, 3, 7] = True
    assert ok.all()


def test_a_million_weights_below_what_fp16_holds_of_one():
    """One position with nearly all weight, 2^20 others with 2^-25.3 of it each: together a fortieth, and their values are the opposite of its.  (Errors in the
    mean of the columns, measured: 0.0254 with weights of at most 1, which all are cut off, 0.0108 with the factor of 2^4, 0.0088 with weights in bf16.)"""
    n, lay = 2 ** 20, dict(heads=1, dn=16, dr=64, dv=16, dl=128)
    b = Batch(lay, [2], [n], form=edg.LATENT_EXPANDED, page=256)
    u = torch.randn(128, generator=torch.Generator().manual_seed(9)).bfloat16().cuda()
    b.cache.zero_()
    b.cache[..., :128] = u
    one = (int(b.table[0, 1]), 44)                              # position 300
    b.cache[one][:128] = -u
    b.cache[one][128] = 9.8125
    b.q_buf.zero_()
    b.q_rope.zero_()
    b.q_rope[:, :, 0] = 16.0
    b.attend()
    torch.cuda.synchronize()
    assert edg.workspace_status(b.ws) == 0
    share = (n - 1) * 2.0 ** -(80 ** -0.5 * 16.0 * 9.8125 / math.log(2.0))
    assert 0.02 < share < 0.03
    want = -(b.W_uv.double() @ u.double()) * (1 - share) / (1 + share)
    # Its weight and value are rounded by 2^-11 each, the others' weights of 2^(4 - 25.3) are held to 2^-25, an eighth of them; y by 2^-8.  Their products are added to an
    # fp32 sum that holds the one's from the third tile on: an addend below 2^-24 of a 32-bit sum may be lost whole, and so may n of them, which is more
    # than all of these together -- a bound for 32-bit sums, whatever the weights' type.
    tol = 2.0 ** -8 + 2.0 ** -10 + share * 2.0 ** -3 + n * 2.0 ** -24
    off = (b.y.double() - want).abs() / want.abs()
    assert (off <= tol).all()
