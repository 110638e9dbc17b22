"""GPU tests of tva_chunk_attn against the definition in 64 bits (oracle/layer_oracle.py)."""
import numpy as np
import pytest

from oracle import cache_oracle, fp8_oracle, layer_oracle as orc
from tests import cache_cases as cc

pytestmark = pytest.mark.gpu
bf16, to_bf16 = cache_oracle.bf16, cache_oracle.to_bf16


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


H = {"4/4/64": (4, 4, 64), "24/8/128": (24, 8, 128), "32/8/128": (32, 8, 128), "32/8/64": (32, 8, 64), "16/1/128": (16, 1, 128), "5/5/128": (5, 5, 128),
     "71/1/64": (71, 1, 64)}


def make(rng, lay, total, rows):
    """A cache of random rows; rows of no sequence hold NaN.  -> tensors for make_cache, values of positions"""
    D = lay.D
    if rows == "bf16":
        k, v = (np.full((lay.rows, D), 0x7FC0, np.uint16) for _ in range(2))
        for b, n in enumerate(total):
            at = lay.at(b, np.arange(n))
            k[at], v[at] = (to_bf16(rng.standard_normal((*at.shape, D))) for _ in range(2))
        return dict(kind=0, k=k, v=v), lambda x, b, n: bf16(x[lay.at(b, np.arange(n))])
    k, v = (np.full((lay.rows, D), 0x7F, np.uint8) for _ in range(2))
    for b, n in enumerate(total):
        at = lay.at(b, np.arange(n))
        for x in (k, v):
            c = rng.integers(0, 256, (*at.shape, D)).astype(np.uint8)
            x[at] = np.where((c & 0x7F) >= 0x60, c & 0x9F, c)  # values up to 15
    return dict(kind=1, k=k, v=v, k_scale=0.125, v_scale=0.25), lambda x, b, n: fp8_oracle.e4m3_decode(x[lay.at(b, np.arange(n))]) * (0.125 if x is k else 0.25)


def compare(out, lse, ro, rl, size, reach, weight_step):
    """A weight is rounded to bf16 once as a factor of V (half a step, 2^-8; with its remainder 2^-16), out once more; scores are fp32 sums of
    D products and the exponentials' arguments are fp32 numbers of the size of scale * sum |q| |k|: 2^-20 of it, over all."""
    e = 2.0 ** -20 * (reach + 1 + np.abs(np.where(np.isfinite(rl), rl, 0)))
    fine = np.isfinite(rl)
    assert np.array_equal(np.isneginf(lse), np.isneginf(rl))
    assert (np.abs(lse - rl)[fine] <= e[fine]).all(), np.abs(lse - rl)[fine].max()
    tol = 1.01 * (weight_step * size + 2.0 ** -8 * np.abs(ro)) + (2 * e[..., None] + 2.0 ** -18) * size + 1e-30
    ok = np.isfinite(ro)
    assert not ((ok != np.isfinite(out)) | (np.isnan(ro) != np.isnan(out))).any()
    assert (np.abs(out - ro)[ok] <= tol[ok]).all(), (np.abs(out - ro)[ok] / tol[ok]).max()
    inf = np.isinf(ro)
    assert np.array_equal(out[inf], ro[inf])


def _attend(torch, rng, heads, sizes, lengths, page=0, head_major=False, rows="bf16", window=0, n_first=0, tree=None, splits=0, plan=0, scale=None,
            room=None, change=None, spare_q=0, max_T=None, max_L=None, padded=0, stream=None, lse_wanted=True):
    from paper_2510_26577_amd import chunk
    Hq, Hkv, D = heads
    B = len(sizes)
    total = [L + T for L, T in zip(lengths, sizes)]
    lay = cc.Layout(rng, total if room is None else room, Hkv, D, page, head_major)
    held, values = make(rng, lay, total if room is None else [min(a, b) for a, b in zip(total, room)], rows)
    if change is not None:
        change(held, lay)
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n = int(cu[-1])
    sets = None if tree is None else [cc.ancestor_sets(p) for p in cc.trees(rng, sizes)] if tree is True else tree
    scale = D ** -0.5 if scale is None else scale
    q = to_bf16(rng.standard_normal((n + padded, Hq, D)))
    dq = cc.dev(np.concatenate([q.reshape(n + padded, -1), np.full((n + padded, 8 * spare_q), 0x7FC0, np.uint16)], 1))[:, :Hq * D].unflatten(1, (Hq, D))
    out = torch.full((n + padded + 1, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + padded + 1, Hq), 7.0, device="cuda") if lse_wanted else None
    mask = None
    if sets is not None:
        words = 1 + (max(sizes) > 64)
        mask = np.concatenate([cc.mask_words(s, words) for s in sets] + [np.zeros((padded, words), np.uint64)])
    tensors = {name: cc.dev(x) if isinstance(x, np.ndarray) else x for name, x in held.items()}
    args = chunk.make_args(q=dq, cache=lay.cache(**tensors), cu_T=cc.dev(cu), L=cc.dev(np.array(lengths, np.int32)), Hkv=Hkv, max_T=max(sizes) if max_T is None else max_T,
                           max_L=max(lengths) if max_L is None else max_L, scale=scale, window=window, n_first=n_first,
                           anc_mask=None if mask is None else cc.dev(mask), out=out, lse=lse, num_splits=splits, plan_rows=plan)
    ws = chunk.attn_workspace(args, "cuda")
    if ws is not None:
        ws.fill_(float("nan"))
    torch.cuda.synchronize()
    chunk.attn_raw(args, stream)
    torch.cuda.synchronize()
    got = bf16(cc.bits(out))
    got_lse = lse.double().cpu().numpy() if lse_wanted else None
    assert (got[n:] == 7).all() and (not lse_wanted or (got_lse[n:] == 7).all())  # behind the last row
    for b in range(B):
        r, end = slice(cu[b], cu[b + 1]), total[b] if room is None else min(total[b], lay.table.shape[1] * page if page else room[b])
        ok, _ = orc.seen(lengths[b], sizes[b], window, n_first, None if sets is None else sets[b], end)
        with np.errstate(invalid="ignore"):
            K, V = values(held["k"], b, end), values(held["v"], b, end)
            ro, rl, size, reach = orc.attention(bf16(q[r]), K, V, ok[:, :end], scale)
        compare(got[r], got_lse[r] if lse_wanted else rl, ro, rl, size, reach, 2.0 ** -16 if chunk.plan_rows(args) == 32 else 2.0 ** -8)
    return args


@pytest.mark.parametrize("heads", list(H))
@pytest.mark.parametrize("page,head_major", [(0, False), (0, True), (16, False), (48, True), (5, False)])
def test_chunks_over_heads_and_layouts(torch, heads, page, head_major):
    _attend(torch, np.random.default_rng(1), H[heads], [13, 1, 30], [150, 3, 64], page, head_major)


@pytest.mark.parametrize("L", [0, 1, 31, 63, 64, 65, 127, 129, 320])
@pytest.mark.parametrize("T", [1, 2, 17, 33, 70, 200])
def test_chunks_over_lengths(torch, T, L):
    _attend(torch, np.random.default_rng(L + T), H["32/8/128"], [T], [L], 16 if L % 2 else 0)


@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
@pytest.mark.parametrize("plan", [32, 128, 256])
@pytest.mark.parametrize("D,page", [(64, 0), (128, 0), (128, 16), (64, 24)])
@pytest.mark.parametrize("splits", [1, 3])
def test_chunks_with_rows_named(torch, rows, plan, D, page, splits):
    """Every size of a workgroup, with chunks that fill part of one, one, and several."""
    _attend(torch, np.random.default_rng(plan), (12, 2, D), [70, 1, 6, 150, 0, 22], [333, 40, 64, 200, 9, 0], page, rows=rows, splits=splits, plan=plan)


@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
@pytest.mark.parametrize("plan", [32, 128, 256])
@pytest.mark.parametrize("window,n_first", [(1, 0), (1, 3), (7, 0), (64, 4), (65, 1), (100, 70), (300, 200), (1000, 2), (1 << 30, 5)])
def test_windows(torch, rows, plan, window, n_first):
    rng = np.random.default_rng(window)
    _attend(torch, rng, (8, 2, 128 if plan % 128 else 64), [130, 1, 40, 5], [500, 700, 0, 66], 16, rows=rows, window=window, n_first=n_first, plan=plan, splits=0 if window % 2 else 4)


@pytest.mark.parametrize("T", [1, 8, 63, 64, 65, 97, 128])
@pytest.mark.parametrize("plan", [0, 32, 128, 256])
def test_trees(torch, T, plan):
    _attend(torch, np.random.default_rng(T), H["24/8/128"], [T, 1, T // 2], [70, 0, 200], 16, tree=True, plan=plan)


@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
@pytest.mark.parametrize("window,n_first", [(1, 0), (2, 0), (3, 1), (5, 80), (40, 4), (200, 0), (200, 300)])
@pytest.mark.parametrize("D", [64, 128])
def test_trees_in_windows(torch, rows, window, n_first, D):
    """Windows that end among the ancestors, and first tokens that reach into the tree."""
    for plan in (0, 32, 256):
        _attend(torch, np.random.default_rng(window), (8, 2, D), [60, 1, 100, 7], [70, 90, 500, 0], 0, rows=rows, window=window, n_first=n_first, tree=True, plan=plan)


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_in_splits(torch, splits, D):
    _attend(torch, np.random.default_rng(splits), (8, 2, D), [9, 140, 3, 1], [1000, 130, 0, 64], 16, splits=splits)
    _attend(torch, np.random.default_rng(splits), (8, 2, D), [9, 140, 3, 1], [1000, 130, 0, 64], 16, splits=splits, window=90, n_first=5)


def test_many_sequences(torch):
    rng = np.random.default_rng(8)
    for B in (64, 65, 200):
        sizes, lengths = rng.integers(0, 4, B), rng.integers(0, 300, B)
        sizes[B // 2] = 50
        _attend(torch, rng, (8, 2, 64), sizes.tolist(), lengths.tolist(), 16)


def test_sequences_without_tokens_and_padded_rows(torch):
    rng = np.random.default_rng(9)
    _attend(torch, rng, (8, 2, 128), [0, 3, 0, 50, 0], [10, 0, 5, 100, 3], 16, padded=40)
    _attend(torch, rng, (8, 2, 128), [0, 3, 0, 50, 0], [10, 0, 5, 100, 3], 0, padded=7, tree=True, spare_q=2)


def test_masks_that_leave_a_row_empty(torch):
    """A node without itself or an ancestor: it sees what is cached of its window, or nothing."""
    rng = np.random.default_rng(10)
    sets = [np.zeros((6, 6), bool), cc.ancestor_sets(cc.trees(rng, [4])[0])]
    sets[0][2, 2] = sets[0][3, 1] = True
    for lengths in ([0, 0], [0, 50], [50, 0], [200, 3]):
        for splits in (1, 2):
            for window in (0, 1, 10):
                _attend(torch, rng, H["24/8/128"], [6, 4], lengths, tree=sets, splits=splits, window=window)


@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
@pytest.mark.parametrize("plan", [32, 128, 256])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(torch, rows, plan):
    rng = np.random.default_rng(11)
    nan, inf, ninf = (0x7FC0, 0x7F80, 0xFF80) if rows == "bf16" else (0x7F, 0xFF, 0x7F)

    def change(held, lay):
        at = lay.at(0, np.arange(260))
        held["v"][at[230, 0], 3], held["v"][at[231, 1], 60], held["v"][at[205, 1], 7] = nan, inf, ninf
        held["v"][at[3, 0], 9] = nan      # leaves the window
        held["k"][at[240, 0], 5] = nan
        held["k"][at[259]] = nan          # the last token's key, seen by itself alone
        at = lay.at(1, np.arange(33))
        held["v"][at[32]] = nan

    for kw in (dict(), dict(window=40), dict(window=30, n_first=2), dict(splits=3)):
        _attend(torch, rng, (8, 2, 64), [60, 33], [200, 0], 16, rows=rows, plan=plan, change=change, **kw)
    _attend(torch, rng, (8, 2, 64), [60, 33], [200, 0], 16, rows=rows, plan=plan, change=change, tree=True, window=50)


def test_scores_that_are_large(torch):
    """Softmax weights of one key, and references that move in every tile."""
    rng = np.random.default_rng(12)

    def growing(held, lay):
        at = lay.at(0, np.arange(700))
        held["k"][at] = to_bf16(bf16(held["k"][at]) * np.linspace(0.1, 30, 700)[:, None, None])

    for plan in (32, 128, 256):
        _attend(torch, rng, (8, 2, 128), [100], [600], 16, scale=1.0, plan=plan, change=growing)
        _attend(torch, rng, (8, 2, 128), [100], [600], 16, scale=1e-30, plan=plan)


@pytest.mark.parametrize("page", [0, 16])
def test_positions_without_a_place_are_not_read(torch, page):
    rng = np.random.default_rng(13)
    _attend(torch, rng, (8, 2, 64), [40, 5], [30, 7], page, room=[48, 48])
    _attend(torch, rng, (8, 2, 64), [40, 5], [70, 7], page, room=[48, 48], window=20)
    _attend(torch, rng, (8, 2, 64), [40, 5], [30, 7], page, room=[48, 48], tree=True)


def test_bounds_that_are_larger_and_smaller_than_need_be(torch):
    rng = np.random.default_rng(14)
    for max_L in (0, 10, 100000):
        _attend(torch, rng, (8, 2, 64), [40, 5], [900, 7], 16, max_L=max_L)
    for max_T in (41, 200, 3000):
        _attend(torch, rng, (8, 2, 64), [40, 5], [30, 7], 16, max_T=max_T)
    _attend(torch, rng, (8, 2, 64), [40, 5], [30, 7], 16, lse_wanted=False)


def test_rows_beyond_the_bound_are_not_computed(torch):
    from paper_2510_26577_amd import chunk
    rng = np.random.default_rng(15)
    lay = cc.Layout(rng, [60], 2, 64)
    held, _ = make(rng, lay, [60], "bf16")
    q = cc.dev(to_bf16(rng.standard_normal((50, 4, 64))))
    out = torch.full((50, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    c = lay.cache(**{n: cc.dev(x) if isinstance(x, np.ndarray) else x for n, x in held.items()})
    chunk.attn(q, c, cc.dev([0, 50], np.int32), cc.dev([10], np.int32), Hkv=2, max_T=20, max_L=10, scale=0.1, out=out)
    assert (out[20:] == 7).all() and not (out[:20] == 7).all(-1).any()


def test_one_long_chunk(torch):
    _attend(torch, np.random.default_rng(16), (8, 2, 128), [1100], [900], 64)
    _attend(torch, np.random.default_rng(17), (4, 1, 64), [1500], [37], 16, window=333, n_first=4, rows="e4m3")


@pytest.mark.parametrize("plan", [32, 128, 256])
@pytest.mark.parametrize("B,kind", [(2, "alone"), (5, "alone"), (64, "alone"), (65, "alone"), (12, "even"), (9, "ragged"), (64, "ragged"), (66, "ragged"), (7, "bounded")])
def test_blocks_of_batches(torch, B, kind, plan):
    """Row blocks are numbered by keys, evenly or by rows: each is computed once, whatever the sequences' lengths."""
    rng = np.random.default_rng(1000 * B + plan)
    sizes, lengths, more = rng.integers(1, 40, B), rng.integers(0, 200, B), {}
    if kind == "alone":  # all but one have no tokens
        sizes[:] = 0
        sizes[rng.integers(B)] = 150
    elif kind == "even":
        sizes[:], lengths[::2] = 70, 33
    elif kind == "ragged":
        sizes[rng.integers(0, B, 3)] = 0, 131, 97
        lengths[:3] = 180  # (keys alike)
    else:
        more = dict(max_T=500, padded=800)
    _attend(torch, rng, (4, 1, 64), sizes.tolist(), lengths.tolist(), 16, plan=plan, splits=1 + B % 3, **more)
