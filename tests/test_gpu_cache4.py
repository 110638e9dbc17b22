"""GPU parity of the 4-bit rows (include/tva_cache.h): store and load exact, the attention against 64 bits."""
import sys

import numpy as np
import pytest

from oracle import cache_oracle as orc
from tests import cache_cases as cc

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2510_26577_amd import binding
    binding.load_library()
    return torch


# ---- rows ----
def _rows(rng, shape):
    """bf16 patterns of rows: normal ones of many sizes, and every kind of number."""
    x = orc.to_bf16(rng.standard_normal(shape) * 2.0 ** rng.integers(-20, 20, (*shape[:-1], 1)))
    odd = rng.random(shape) < 0.02
    x[odd] = rng.integers(0, 1 << 16, int(odd.sum())).astype(np.uint16)
    x[rng.random(shape) < 0.1] = 0
    return x


STORES = [  # D, Hkv, sizes, lengths, path lengths (None: all rows), page, head_major, layers
    (128, 8, [60, 8, 1, 33], [100, 0, 7, 31], [5, 0, 1, 9], 0, False, 1),
    (128, 8, [60, 8, 1, 33], [100, 0, 7, 31], [5, 2, 1, 9], 16, False, 3),
    (128, 1, [5], [17], None, 5, True, 1),
    (64, 3, [7, 0, 65], [0, 4, 63], None, 0, True, 2),
    (64, 4, [12, 12], [3, 64], [12, 1], 64, True, 2),
]


@pytest.mark.parametrize("D,Hkv,sizes,lengths,path_len,page,head_major,layers", STORES)
def test_rows_are_stored_and_read_back(torch, D, Hkv, sizes, lengths, path_len, page, head_major, layers):
    from paper_2510_26577_amd import cache4
    say(f"[case] store D={D} Hkv={Hkv} sizes={sizes} path={path_len} page={page}")
    rng = np.random.default_rng(D + len(sizes) + layers)
    B, n_rows = len(sizes), sum(sizes)
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    width = max(path_len) if path_len else max(sizes)
    n = path_len or sizes
    lay = cc.Layout(rng, [L + k for L, k in zip(lengths, n)], Hkv, D, page, head_major)
    cache = cc.FourBit(rng, lay, lengths, layers)
    k, v = (_rows(rng, (layers, n_rows, Hkv, D)) for _ in range(2))
    path = np.full((B, width), -1, np.int32)
    for b in range(B):
        path[b, :n[b]] = np.sort(rng.choice(sizes[b], n[b], replace=False)) if path_len else np.arange(n[b])
    flag, L_out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((B,), -7, dtype=torch.int32, device="cuda")
    more = dict(cu_T=cc.dev(cu), L=cc.dev(np.array(lengths, np.int32)), cache=cache.cache, max_rows=width, err_flag=flag, n_layers=layers,
                layer_stride_cache=lay.rows * D, layer_stride_rows=n_rows * Hkv * D)
    if path_len:
        more.update(path=cc.dev(path), path_len=cc.dev(np.array(n, np.int32)))
    cache4.store(k_rows=cc.dev(k), v_rows=cc.dev(v), L_out=L_out, **more)
    want = [x.copy() for x in (cache.k, cache.ks, cache.v, cache.vs)]
    back = [np.full((layers, n_rows, Hkv, D), 0x1234, np.uint16) for _ in range(2)]
    for layer in range(layers):
        for b in range(B):
            rows = cu[b] + path[b, :n[b]]
            at = lay.at(b, lengths[b] + np.arange(n[b])) + layer * lay.rows
            new = orc.encode_rows(k[layer, rows], v[layer, rows])
            for x, y in zip(want, new):
                x[at] = y
            back[0][layer, rows], back[1][layer, rows] = orc.to_bf16(orc.decode_k(*new[:2])), orc.to_bf16(orc.decode_v(*new[2:]))
    torch.cuda.synchronize()
    for name, x, y in zip(("k", "k scale", "v", "v scale"), cache.download(), want):
        assert np.array_equal(x, y), name
    assert L_out.tolist() == [L + m for L, m in zip(lengths, n)] and not flag.item()
    kb, vb = (cc.dev(np.full((layers, n_rows, Hkv, D), 0x1234, np.uint16)) for _ in range(2))
    cache4.load(k_rows=kb, v_rows=vb, **more)
    torch.cuda.synchronize()
    assert np.array_equal(cc.bits(kb), back[0]) and np.array_equal(cc.bits(vb), back[1]) and not flag.item()


def test_every_number_is_rounded_as_defined(torch):
    """All bf16 patterns, each beside another one that sets the scale."""
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(11)
    x = np.zeros((2048, 1, 128), np.uint16)
    x[:, 0, ::4] = np.arange(65536, dtype=np.uint16).reshape(2048, 32)
    x[:, 0, 1::4] = (x[:, 0, ::4].astype(int) + rng.integers(-600, 600, (2048, 32))).clip(0, 65535)
    x[:, 0, 2::4] = rng.permutation(x[:, 0, ::4].reshape(-1)).reshape(2048, 32) & 0xC0FF | 0x3F00  # about 1
    rng.shuffle(x.reshape(2048 * 4, 32), axis=0)
    lay = cc.Layout(rng, [2048], 1, 128)
    cache = cc.FourBit(rng, lay, [0])
    d = cc.dev(x)
    cache4.store(k_rows=d, v_rows=d, cu_T=cc.dev([0, 2048], np.int32), L=cc.dev([0], np.int32), cache=cache.cache, max_rows=2048)
    got, at = cache.download(), lay.at(0, np.arange(2048))
    for name, a, b in zip(("k", "k scale", "v", "v scale"), got, orc.encode_rows(x, x)):
        assert np.array_equal(a[at], b), name


@pytest.mark.parametrize("page", [0, 16])
def test_rows_without_a_place_are_left_out(torch, page):
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(12)
    lay = cc.Layout(rng, [32, 32, 32], 2, 128, page)
    x = cc.dev(_rows(rng, (12, 2, 128)))
    for L, path, bad in (([0, 30, 0], [[0, 1], [0, 1], [2, 3]], 0), ([0, 31, 0], [[0, 1], [0, 1], [2, 3]], 2), ([0, 0, 0], [[0, 4], [0, 1], [2, 3]], 1),
                         ([0, 0, 0], [[0, 1], [0, 1], [-1, 3]], 3), ([-1, 0, 0], [[0, 1], [0, 1], [2, 3]], 1)):
        cache = cc.FourBit(rng, lay, [0, 0, 0])
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        cache4.store(k_rows=x, v_rows=x, cu_T=cc.dev([0, 4, 8, 12], np.int32), L=cc.dev(L, np.int32), cache=cache.cache, max_rows=2,
                     path=cc.dev(path, np.int32), path_len=cc.dev([2, 2, 2], np.int32), err_flag=flag)
        assert flag.item() == bad
        changed = np.nonzero((cache.download()[3] != cache.vs))[0]
        own = {int(r) for b in range(3) for j in range(2) if 0 <= path[b][j] < 4 and 0 <= L[b] + j < 32 for r in lay.at(b, [L[b] + j])[0]}
        assert set(changed.tolist()) == own


def test_lengths_are_written_without_rows_too(torch):
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(15)
    lay = cc.Layout(rng, [8, 8], 2, 128)
    cache = cc.FourBit(rng, lay, [3, 5])
    L_out, rows = torch.full((2,), -1, dtype=torch.int32, device="cuda"), cc.dev(_rows(rng, (2, 2, 128)))
    cache4.store(k_rows=rows, v_rows=rows, cu_T=cc.dev([0, 1, 2], np.int32), L=cc.dev([3, 5], np.int32), cache=cache.cache, max_rows=0, L_out=L_out)
    assert L_out.tolist() == [3, 5] and np.array_equal(cache.download()[0], cache.k)


# ---- attention ----
def _attend(torch, rng, heads, sizes, lengths, page=0, head_major=False, splits=0, by_parent=False, scale=None, spread=1.0, mask=None, k_tree=None,
            v_tree=None, q=None, max_L=None, check=True, rows=0):
    from paper_2510_26577_amd import cache4
    Hq, Hkv, D = heads
    B, n = len(sizes), sum(sizes)
    say(f"[case] attention heads={heads} sizes={sizes} lengths={lengths} page={page} head_major={head_major} splits={splits}")
    lay = cc.Layout(rng, lengths, Hkv, D, page, head_major)
    cache = cc.FourBit(rng, lay, lengths, spread=spread)
    parents = cc.trees(rng, sizes)
    seen = [cc.ancestor_sets(p) for p in parents] if mask is None else mask
    words = 1 + (max(sizes) > 64)
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    q = orc.to_bf16(rng.standard_normal((n, Hq, D))) if q is None else q
    k_tree = orc.to_bf16(rng.standard_normal((n, Hkv, D))) if k_tree is None else k_tree
    v_tree = orc.to_bf16(rng.standard_normal((n, Hkv, D))) if v_tree is None else v_tree
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out = torch.full((n + 1, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + 1, Hq), 7.0, device="cuda")
    sets = np.concatenate([cc.mask_words(s, words) for s in seen]) if n else np.zeros((0, words), np.uint64)
    kw = dict(parent=cc.dev(np.concatenate(parents))) if by_parent else dict(anc_mask=cc.dev(sets))
    args = cache4.make_attn_args(q=cc.dev(q), k_tree=cc.dev(k_tree), v_tree=cc.dev(v_tree), cache=cache.cache, cu_T=cc.dev(cu),
                                 L=cc.dev(np.array(lengths, np.int32)), max_T=max(sizes), max_L=max(lengths) if max_L is None else max_L,
                                 scale=scale, out=out, lse=lse, num_splits=splits, plan_rows=rows, **kw)
    ws = cache4.attn_workspace(args, "cuda")
    if ws is not None:
        ws.fill_(float("nan"))
    cache4.tree_verify_attn_raw(args)
    torch.cuda.synchronize()
    got, got_lse = orc.bf16(cc.bits(out)), lse.double().cpu().numpy()
    assert (got[n] == 7).all() and (got_lse[n] == 7).all()  # behind the last row
    if check:
        for b in range(B):
            r = slice(cu[b], cu[b + 1])
            K, V = cache.values(b, np.arange(lengths[b]))
            K, V = np.concatenate([K, orc.bf16(k_tree[r])]), np.concatenate([V, orc.bf16(v_tree[r])])
            see = np.concatenate([np.ones((sizes[b], lengths[b]), bool), seen[b]], 1)
            with np.errstate(invalid="ignore"):
                ro, rl, size, reach = orc.attention(orc.bf16(q[r]), K, V, see, scale)
            compare(got[r], got_lse[r], ro, rl, size, reach)
    return args, cache, out[:n], lse[:n]


def compare(out, lse, ro, rl, size, reach):
    """Weights times V's scale are rounded to bf16 once (half a step, 2^-8, of each term), out once more; scores are fp32 sums of
    D products and the exponentials' arguments are fp32 numbers of the size of scale * sum |q| |k|: 2^-20 of it, over all."""
    e = 2.0 ** -20 * (reach + 1 + np.abs(np.where(np.isfinite(rl), rl, 0)))
    fine = np.isfinite(rl)
    assert np.array_equal(np.isneginf(lse), np.isneginf(rl))
    assert (np.abs(lse - rl)[fine] <= e[fine]).all(), np.abs(lse - rl)[fine].max()
    tol = 2.0 ** -8 * 1.01 * (size + np.abs(ro)) + (2 * e[..., None] + 2.0 ** -18) * size + 1e-30
    ok = np.isfinite(ro)
    assert np.array_equal(ok, np.isfinite(out)) and np.array_equal(np.isnan(ro), np.isnan(out))
    assert (np.abs(out - ro)[ok] <= tol[ok]).all(), (np.abs(out - ro)[ok] / tol[ok]).max()
    inf = np.isinf(ro)
    assert np.array_equal(out[inf], ro[inf])


H = {"4/4/64": (4, 4, 64), "24/8/128": (24, 8, 128), "32/8/128": (32, 8, 128), "32/8/64": (32, 8, 64), "16/1/128": (16, 1, 128), "5/5/128": (5, 5, 128)}


@pytest.mark.parametrize("heads", list(H))
@pytest.mark.parametrize("page,head_major", [(0, False), (0, True), (16, False), (48, True), (5, False)])
def test_attention_over_heads_and_layouts(torch, heads, page, head_major):
    _attend(torch, np.random.default_rng(1), H[heads], [13, 1, 30], [150, 3, 64], page, head_major)


@pytest.mark.parametrize("L", [0, 1, 31, 63, 64, 65, 127, 129, 320, 1500])
@pytest.mark.parametrize("T", [1, 2, 17, 33])
def test_attention_over_lengths(torch, T, L):
    _attend(torch, np.random.default_rng(L + T), H["32/8/128"], [T], [L], 16 if L % 2 else 0)


@pytest.mark.parametrize("T", [8, 63, 64, 65, 96, 97, 128])
@pytest.mark.parametrize("by_parent", [False, True])
def test_attention_over_trees(torch, T, by_parent):
    _attend(torch, np.random.default_rng(T), H["24/8/128"], [T, 1, T // 2], [70, 0, 200], by_parent=by_parent)


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_in_splits(torch, splits, D):
    _attend(torch, np.random.default_rng(splits), (8, 2, D), [9, 40, 3, 1], [1000, 130, 0, 64], 16, splits=splits)


@pytest.mark.parametrize("rows", [32, 64, 128])
@pytest.mark.parametrize("D,page", [(64, 0), (128, 0), (128, 16), (64, 64), (128, 64)])
def test_attention_with_rows_named(torch, rows, D, page):
    """Every size of a workgroup, with trees that fill part of one, one, and several."""
    rng = np.random.default_rng(rows)
    for splits in (0, 3):
        _attend(torch, rng, (12, 2, D), [70, 1, 6, 22], [333, 40, 64, 200], page, splits=splits, rows=rows)


@pytest.mark.parametrize("D,page,head_major", [(64, 0, True), (128, 64, False), (64, 16, False)])
def test_attention_of_many_sequences_dealt_out_together(torch, D, page, head_major):
    """More sequences than are dealt out together (64), of lengths that differ, some without a tree, some without a context."""
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(D)
    lengths = rng.integers(0, 2000, 70).tolist()
    lengths[3], lengths[40], lengths[66] = 0, 2200, 64
    sizes = rng.integers(1, 4, 70).tolist()
    sizes[5] = sizes[63] = 0
    args, *_ = _attend(torch, rng, (8, 8, D), sizes, lengths, page, head_major)
    assert cache4.plan_splits(args) > 20  # (a sequence alone would have one)


def test_attention_of_empty_trees_and_masks_without_keys(torch):
    rng = np.random.default_rng(5)
    _attend(torch, rng, H["32/8/64"], [0, 3, 0, 5, 0], [10, 0, 5, 100, 3])
    seen = [np.zeros((6, 6), bool), cc.ancestor_sets(cc.trees(rng, [4])[0])]
    seen[0][2, 2] = True
    for lengths in ([0, 0], [0, 50], [50, 0]):
        for splits in (1, 2):
            _, _, out, lse = _attend(torch, rng, H["24/8/128"], [6, 4], lengths, mask=seen, splits=splits)
            assert lengths[0] or (not out[0].any() and torch.isneginf(lse[0]).all())


def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(torch):
    rng = np.random.default_rng(6)
    for T in (5, 40, 100):
        v = orc.to_bf16(rng.standard_normal((T, 2, 128)))
        k = orc.to_bf16(rng.standard_normal((T, 2, 128)))
        v[T - 2, 0, 3], v[T - 1, 1, 100], v[T // 2, 1, 7] = 0x7F80, 0xFF80, 0x7FC1
        k[T - 1] = 0x7FC0  # a leaf's key, seen by the leaf alone
        seen = [cc.ancestor_sets(np.arange(-1, T - 1, dtype=np.int32))]
        seen[0][T - 1] = False
        seen[0][:, T - 1] = False
        _attend(torch, rng, (8, 2, 128), [T], [70], mask=seen, v_tree=v, k_tree=k)


def test_attention_of_rows_that_are_nan(torch):
    """A query that is NaN gives NaN, and to itself alone."""
    rng = np.random.default_rng(7)
    q = orc.to_bf16(rng.standard_normal((9, 8, 128)))
    q[4, 3, 50] = 0x7FC0
    for splits in (1, 4):
        _, _, out, lse = _attend(torch, rng, (8, 2, 128), [9], [400], q=q, splits=splits, check=False)
        bad = torch.isnan(out).all(-1)
        assert bad[4, 3] and int(bad.sum()) == 1 and int(torch.isnan(out).any(-1).sum()) == 1
        assert torch.isnan(lse[4, 3]) and int(torch.isnan(lse).sum()) == 1


def test_attention_of_scores_far_apart(torch):
    rng = np.random.default_rng(8)
    _attend(torch, rng, H["32/8/128"], [20], [500], spread=8.0, scale=0.5)
    _attend(torch, rng, H["32/8/128"], [20], [500], spread=2.0 ** -20)


def test_context_is_cut_where_the_bound_says(torch):
    rng = np.random.default_rng(9)
    a, cache, out, lse = _attend(torch, rng, (8, 2, 128), [4], [300], max_L=100, check=False)
    q, kt, vt = (orc.bf16(cc.bits(t)) for t in (a._keep[2], a._keep[3], a._keep[4]))
    K, V = cache.values(0, np.arange(100))
    seen = cc.mask_words  # (the tree's own sets, back from the words)
    words = a._keep[5].cpu().numpy().view(np.uint64)
    tree = np.array([[bool(w[0] >> np.uint64(j) & np.uint64(1)) for j in range(4)] for w in words])
    ref = orc.attention(q, np.concatenate([K, kt]), np.concatenate([V, vt]), np.concatenate([np.ones((4, 100), bool), tree], 1), a.scale)
    compare(orc.bf16(cc.bits(out)), lse.double().cpu().numpy(), *ref)


def test_attention_in_a_graph_on_a_stream_of_its_own(torch):
    """Captured once, replayed with other inputs in the same buffers, eager calls of the program between."""
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(10)
    args, cache, out, lse = _attend(torch, rng, H["32/8/128"], [8, 20], [700, 90], 16, splits=5)
    want = (out.clone(), lse.clone())
    q = args._keep[2]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            cache4.tree_verify_attn_raw(args)
    for i in range(4):
        x = torch.randn_like(q.float()).to(torch.bfloat16) if i else None
        if i:
            q.copy_(x)
            cache4.tree_verify_attn_raw(args)
            torch.cuda.synchronize()
            want = (out.clone(), lse.clone())
        out.fill_(3.0), lse.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_attention_far_into_a_large_pool(torch):
    """Rows whose byte offsets pass 32 bits."""
    from paper_2510_26577_amd import cache4
    rng = np.random.default_rng(13)
    Hq, Hkv, D, page, L, T = 8, 2, 128, 16, 100, 3
    pages = (9 << 29) // (64 * Hkv * page)  # 4.5 GiB of K
    small = cc.Layout(rng, [L], Hkv, D, page)
    cache = cc.FourBit(rng, small, [L])
    n = -(-L // page)
    far = np.arange(pages - n, pages, dtype=np.int32)[::-1].copy()
    big = dict(k=torch.empty((pages * page * Hkv, 64), dtype=torch.uint8, device="cuda"), v=torch.empty((pages * page * Hkv, 64), dtype=torch.uint8, device="cuda"),
               k_row_scale=torch.empty((pages * page * Hkv, 4), dtype=torch.uint8, device="cuda"),
               v_row_scale=torch.empty(pages * page * Hkv, dtype=torch.bfloat16, device="cuda"))
    for i in range(n):
        a, b = int(small.table[0, i]) * page * Hkv, int(far[i]) * page * Hkv
        for name in big:
            big[name][b:b + page * Hkv] = cache.d[name][a:a + page * Hkv]
    q, kt, vt = (cc.dev(orc.to_bf16(rng.standard_normal((T, h, D)))) for h in (Hq, Hkv, Hkv))
    kw = dict(cu_T=cc.dev([0, T], np.int32), L=cc.dev([L], np.int32), max_T=T, max_L=L, scale=0.1, parent=cc.dev([-1, 0, 0], np.int32))
    near = cache4.tree_verify_attn(q, kt, vt, cache.cache, **kw)
    far_c = cache4.make_cache(**big, page_table=cc.dev(far[None]), page_size=page)
    got = cache4.tree_verify_attn(q, kt, vt, far_c, **kw)
    assert torch.equal(near[0], got[0]) and torch.equal(near[1], got[1])
    # and stored there
    rows = cc.dev(orc.to_bf16(rng.standard_normal((L, Hkv, D))))
    for c in (cache.cache, far_c):
        cache4.store(k_rows=rows, v_rows=rows, cu_T=cc.dev([0, L], np.int32), L=cc.dev([0], np.int32), cache=c, max_rows=L)
    a, b = cache4.tree_verify_attn(q, kt, vt, cache.cache, **kw), cache4.tree_verify_attn(q, kt, vt, far_c, **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and not torch.equal(a[0], got[0])
