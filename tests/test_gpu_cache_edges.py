"""The paged cache on the GPU: orders of items, ragged tiles and magnitudes that the plain cases do not reach."""
import pytest
import torch

from test_gpu_cache import BF16, E4M3, INT8, Setup, attend, check, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim,group", [(BF16, 64, 1), (BF16, 128, 2), (INT8, 64, 5), (E4M3, 128, 3)])
def test_short_items_behind_items_that_are_cut(dtype, dim, group):
    """Long sequences, most of which lie in several CTAs, each in front of a dozen short ones: a join is followed at once by items that need none.
    Every run gives the same."""
    lens = sum(([700] + [1 + (7 * i + j) % 16 for j in range(12)] for i in range(20)), [])
    s = Setup(dtype, dim, 16, 4, lens)
    s.fill()
    qlens = [1] * len(lens)
    q = rand(s.g, len(lens), 4 * group, dim, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)
    for _ in range(20):
        again = attend(s, qlens, q)
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype", [BF16, INT8, E4M3])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group,tokens", [(1, 17), (1, 131), (3, 43), (7, 20), (11, 13), (100, 1), (48, 5)])
def test_tiles_with_rows_that_do_not_exist(dtype, dim, group, tokens):
    """Warps that have rows of a tile and places without one, in one query tile and in two, in items that are cut and whole ones."""
    lens, qlens = [1500, tokens + 30, tokens], [tokens] * 3
    s = Setup(dtype, dim, 16, 2, lens)
    s.fill()
    q = rand(s.g, 3 * tokens + 2, 2 * group, dim, times=1.5)
    o, lse = attend(s, qlens, q)
    check(s, qlens, q, o, lse)
