"""The int4 projection where a warp takes two tiles of 16 rows at once (some thousand rows): odd numbers of tiles and of rows, each group size.

Tolerances are those of test_gpu_linear."""
import pytest

from test_gpu_linear import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [6113, 6129, 6144])             # 383 tiles, 384 with one row in the last, 384
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,rank,out", [(1, 0, "f32"), (1, 16, "bf16"), (16, 0, "bf16"), (40, 33, "f32"), (64, 16, "f16")])
def test_two_row_tiles_at_once(N, group, T, rank, out):
    c = Case(N, 2048, group, rank, T, out)
    c.run()
    c.check()


@pytest.mark.parametrize("N,K,T", [(17, 256, 64), (2047, 2048, 64), (40001, 256, 16), (40001, 128, 3), (33, 65536, 2)])
def test_shapes_of_a_launch(N, K, T):
    """Few rows for many tokens, many rows with few blocks each, one pair of tiles over the longest input."""
    c = Case(N, K, 64, 8, T)
    c.run()
    c.check()
    first = c.y.clone()
    c.run()
    c.check()
    assert first.equal(c.y)
