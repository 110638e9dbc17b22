"""How often the attention over 4-bit rows rounds (include/tva_cache.h): against 64 bits, with what is left of a softmax weight's
rounding where few keys share a row and where many do."""
import numpy as np
import pytest

from oracle import cache_oracle as orc
from tests import cache_cases as cc
from tests.test_gpu_cache4 import _attend, torch  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _reference(args, cache, lengths, sizes):
    """Per row and head: out, lse, sum p |v|, the part of it whose weights may be rounded to bf16 (cached keys with at most an eighth of
    the row), and the largest scale * sum |q| |k|."""
    cu = np.concatenate([[0], np.cumsum(sizes)])
    q, kt, vt = (orc.bf16(cc.bits(args._keep[i])) for i in (2, 3, 4))
    words = args._keep[5].cpu().numpy().view(np.uint64)
    G = args.Hq // args.Hkv
    out, size, light = (np.zeros(q.shape) for _ in range(3))
    lse, reach = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    for b, L in enumerate(lengths):
        K, V = cache.values(b, np.arange(L))
        for i in range(cu[b], cu[b + 1]):
            sees = [j for j in range(sizes[b]) if int(words[i, j // 64]) >> (j % 64) & 1]
            rows = cu[b] + np.array(sees, int)
            for h in range(args.Hq):
                k, v = np.concatenate([K[:, h // G], kt[rows, h // G]]), np.concatenate([V[:, h // G], vt[rows, h // G]])
                x = args.scale * (k @ q[i, h])
                lse[i, h] = np.log(np.exp(x - x.max()).sum()) + x.max()
                p = np.exp(x - lse[i, h])
                out[i, h], size[i, h] = p @ v, p @ np.abs(v)
                rounded = (p <= 0.125 * 1.001) & (np.arange(len(p)) < L)
                light[i, h] = (p * rounded) @ np.abs(v)
                reach[i, h] = args.scale * (np.abs(k) @ np.abs(q[i, h])).max()
    return out, lse, size, light, reach


def _compare(got, ref, light):
    """out is rounded once, half a step: 2^-8.  Scores' sums and exponentials: 2^-20 of their size (test_gpu_cache4.compare).  What
    two roundings to bf16 leave of a weight, 2^-17, with twice that for the fp32 sums: 2^-16 of the row; 2^-8 of what may have one."""
    out, lse, size, may, reach = ref
    e = 2.0 ** -20 * (reach + 1 + np.abs(lse))
    off = (2 * e[..., None] + 2.0 ** -16) * size + (2.0 ** -8 * may if light else 0)
    tol = 2.0 ** -8 * (np.abs(out) + off) + off
    d = np.abs(orc.bf16(cc.bits(got)) - out)
    assert (d <= tol).all(), ((d / tol).max(), int((d > tol).sum()))


@pytest.mark.parametrize("heads", [(24, 8, 128), (32, 8, 64), (4, 4, 64)])
@pytest.mark.parametrize("page", [0, 16, 64])
def test_rows_of_few_keys_are_rounded_once(torch, heads, page):
    """Up to seven keys: the largest weight is more than an eighth of its row, in whichever tile."""
    rng = np.random.default_rng(heads[0] + page)
    lengths = rng.integers(0, 7, 24).tolist()
    for scale in (0.02, 1.0 / np.sqrt(heads[2]), 0.5):
        args, cache, out, _ = _attend(torch, rng, heads, [1] * 24, lengths, page, scale=scale, check=False)
        _compare(out, _reference(args, cache, lengths, [1] * 24), False)


@pytest.mark.parametrize("D,page,T,rows,splits", [(128, 0, 1, 0, 0), (128, 16, 1, 0, 1), (128, 64, 3, 0, 3), (64, 16, 2, 32, 2), (128, 16, 17, 64, 1), (64, 0, 17, 64, 2),
                                                  (128, 0, 33, 128, 1), (64, 64, 33, 128, 2)])
def test_heavy_weights_of_long_rows_are_not_rounded(torch, D, page, T, rows, splits):
    """Scores of a spread at which one key, or a few, hold most of a row, wherever in the context."""
    rng = np.random.default_rng(D + page + T)
    lengths = [700, 130]
    heavy = 0
    for scale in (2.0, 6.0):
        args, cache, out, _ = _attend(torch, rng, (8, 2, D), [T, T], lengths, page, splits=splits, rows=rows, scale=scale / np.sqrt(D), check=False)
        ref = _reference(args, cache, lengths, [T, T])
        heavy += int((ref[3].sum(-1) < 0.5 * ref[2].sum(-1)).sum())
        _compare(out, ref, True)
    assert heavy > T  # (rows with most of their weight in few keys)


@pytest.mark.parametrize("D,page", [(128, 0), (128, 16), (64, 64), (64, 5)])
def test_blocks_of_32_rows_round_once(torch, D, page):
    """Several blocks of 32 rows, the form of short work: no weight is rounded to bf16 alone."""
    rng = np.random.default_rng(D + page)
    lengths, sizes = [300, 64, 1], [20, 9, 13]
    for splits in (0, 2):
        args, cache, out, _ = _attend(torch, rng, (8, 2, D), sizes, lengths, page, splits=splits, rows=32, check=False)
        _compare(out, _reference(args, cache, lengths, sizes), False)


def test_tree_values_are_rounded_once(torch):
    """A tree without a context, by every number of nodes a row sees: bf16 values under fp32 weights."""
    rng = np.random.default_rng(3)
    for T in (9, 64, 100):
        seen = [np.tri(T, dtype=bool)]
        args, cache, out, _ = _attend(torch, rng, (8, 2, 128), [T], [0], mask=seen, check=False)
        _compare(out, _reference(args, cache, [0], [T]), False)
