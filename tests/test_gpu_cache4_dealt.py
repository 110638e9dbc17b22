"""The attention over 4-bit rows where several sequences' keys are dealt out together (include/tva_cache.h), with trees of several row
blocks: the blocks of one head deal out different sequences, since trees that end before a block have no keys in it."""
import numpy as np
import pytest

from tests.test_gpu_cache4 import _attend, torch  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _batch(rng, B, max_T):
    """Trees of all sizes, some empty, some of one node, and contexts of which a few are long."""
    sizes = rng.integers(0, max_T + 1, B)
    sizes[0], sizes[B // 2], sizes[B // 3], sizes[-1] = max_T, 0, 1, max_T - 1
    sizes[1:4] = 0, max_T // 3, max_T
    lengths = rng.integers(0, 500, B)
    lengths[[0, 5, B - 2]] = 2100, 1999, 2050
    lengths[[2, B // 2 + 1]] = 0, 64
    return sizes.tolist(), lengths.tolist()


@pytest.mark.parametrize("page,head_major", [(0, False), (16, False), (64, True)])
@pytest.mark.parametrize("D,rows,B,max_T", [(128, 64, 33, 48), (128, 128, 25, 40), (64, 64, 33, 48), (64, 128, 70, 70), (128, 32, 63, 20), (64, 32, 63, 20)])
def test_row_blocks_deal_out_the_sequences_that_reach_them(torch, D, rows, B, max_T, page, head_major):
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(D + rows + page)
    sizes, lengths = _batch(rng, B, max_T)
    args, *_ = _attend(torch, rng, (8, 2, D), sizes, lengths, page, head_major, rows=rows, by_parent=page == 16)
    blocks, groups = -(-max_T * 4 // rows), -(-B // 64)
    assert blocks > 1 and cache4.plan_splits(args) == 512 // (2 * blocks * groups)  # (a sequence by itself: 256 / (2 * blocks * B), or 1)


def test_the_library_deals_out_long_trees_by_itself(torch):
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(9)
    sizes, lengths = _batch(rng, 40, 48)
    args, *_ = _attend(torch, rng, (8, 2, 128), sizes, lengths, 16)
    assert cache4.plan_splits(args) > 20


@pytest.mark.parametrize("page", [0, 5, 16, 64])
@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 2, 64), (3, 3, 128)])
def test_heads_kept_together_in_more_than_the_last_level_cache_holds(torch, heads, page):
    """One block of rows per head, head-major, and a bound of the lengths by which the cache passes 256 MB: keys are read another way then."""
    rng = np.random.default_rng(heads[0] + page)
    assert 3 * (1 << 20) * heads[1] * heads[2] > 256 << 20
    for sizes, lengths in (([1, 1, 1], [700, 0, 64]), ([5, 0, 8], [130, 64, 2100]), ([2, 3, 1], [1, 63, 65])):
        _attend(torch, rng, heads, sizes, lengths, page, True, max_L=1 << 20)
    _attend(torch, rng, heads, [7], [900], page, True, max_L=1 << 22, splits=3)
