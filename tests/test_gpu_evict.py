"""GPU parity of eviction (include/tva_cache.h): weights of keys against 64 bits, choice and moves exact, and a run of the
operators together with the attention over 4-bit rows."""
import sys

import numpy as np
import pytest

from oracle import cache_oracle as orc
from tests import cache_cases as cc
from tests.test_gpu_cache4 import compare

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


def _e4m3(rng, shape):
    import torch
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.float8_e4m3fn)
    return x.view(torch.uint8).cuda(), x.double().numpy()


WEIGHTS = [  # heads, sizes, path lengths (None: all), lengths after the commit, rows, page, head_major
    ((32, 8, 128), [16, 60, 9], [3, 1, 9], [300, 1, 129], "e2m1", 16, False),
    ((32, 8, 128), [16, 60, 9], [3, 0, 9], [300, 40, 9], "bf16", 0, False),
    ((24, 8, 128), [5, 5], [5, 2], [64, 33], "e4m3", 32, True),
    ((4, 4, 64), [12], [4], [31], "bf16", 5, False),
    ((32, 8, 64), [40, 1, 0], None, [40, 200, 17], "e2m1", 0, True),
    ((16, 1, 128), [70], None, [500], "e4m3", 0, False),
    ((16, 1, 128), [300], None, [333], "e2m1", 48, True),
]


@pytest.mark.parametrize("heads,sizes,path_len,lengths,rows,page,head_major", WEIGHTS)
def test_key_weights(torch, heads, sizes, path_len, lengths, rows, page, head_major):
    from paper_2510_26577_amd import cache4, evict
    say(f"[case] weights heads={heads} sizes={sizes} path={path_len} lengths={lengths} rows={rows}")
    rng = np.random.default_rng(len(sizes) + lengths[0])
    Hq, Hkv, D = heads
    B, n_rows = len(sizes), sum(sizes)
    lay = cc.Layout(rng, lengths, Hkv, D, page, head_major)
    if rows == "e2m1":
        four = cc.FourBit(rng, lay, lengths)
        cache, values, factor = four.cache, lambda b: four.values(b, np.arange(lengths[b]))[0], 1.0
    elif rows == "e4m3":
        d, x = _e4m3(rng, (lay.rows, D))
        factor = 0.37
        cache, values = lay.cache(kind=cache4.ROWS_E4M3, k=d, k_scale=factor), lambda b: x[lay.at(b, np.arange(lengths[b]))] * np.float32(factor)
    else:
        x = orc.to_bf16(rng.standard_normal((lay.rows, D)))
        own = np.zeros(lay.rows, bool)
        for b in range(B):
            own[lay.at(b, np.arange(lengths[b]))] = True
        x[~own] = 0x7FC0
        cache, values = lay.cache(kind=cache4.ROWS_BF16, k=cc.dev(x)), lambda b: orc.bf16(x[lay.at(b, np.arange(lengths[b]))])
    n = path_len or sizes
    width = max(n)
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    path = np.full((B, width), -1, np.int32)
    for b in range(B):
        path[b, :n[b]] = np.sort(rng.choice(sizes[b], n[b], replace=False)) if path_len else np.arange(n[b])
    q = orc.to_bf16(rng.standard_normal((n_rows, Hq, D)))
    lse = (rng.random((n_rows, Hq)) * 3 + 2).astype(np.float32)
    lse[rng.random(lse.shape) < 0.1] = -np.inf
    q[np.isneginf(lse)] = 0x7FC0  # such a row adds nothing, whatever it holds
    ld = max(lengths) + 5
    weight = rng.random((B, Hkv, ld)).astype(np.float32)
    w0 = weight.copy()
    for b in range(B):
        w0[b, :, lengths[b] - n[b]:lengths[b]] = np.nan  # what new entries held does not matter
    dw, dp = cc.dev(w0), cc.dev(np.full((B, Hkv, ld), -3, np.int32))
    kw = dict(path=cc.dev(path), path_len=cc.dev(np.array(n, np.int32))) if path_len else {}
    args = evict.make_key_weight_args(q=cc.dev(q), lse=cc.dev(lse), cache=cache, cu_T=cc.dev(cu), L=cc.dev(np.array(lengths, np.int32)), weight=dw,
                                      max_rows=width, max_L=max(lengths), scale=1.0 / np.sqrt(D), pos=dp, first_pos=cc.dev(np.arange(B) * 1000, np.int32), **kw)
    evict.key_weights_raw(args)
    torch.cuda.synchronize()
    got, pos = dw.cpu().numpy(), dp.cpu().numpy()
    for b in range(B):
        L, r = lengths[b], cu[b] + path[b, :n[b]]
        ref, off = orc.key_weights(weight[b, :, :L], orc.bf16(q[r]), lse[r].astype(np.float64), values(b), n[b], 1.0 / np.sqrt(D))
        # scores are fp32 sums, exponentials' arguments fp32 numbers of the size of scale * sum |q| |k| + |lse|; sums of rows fp32
        tol = 2.0 ** -20 * off + 2.0 ** -22 * (n[b] * Hq // Hkv + 2) * np.abs(ref) + 1e-30
        d = np.abs(got[b, :, :L] - ref)
        assert (d <= tol).all(), (d / tol).max()
        assert np.array_equal(got[b, :, L:], w0[b, :, L:])
        assert (pos[b, :, :L - n[b]] == -3).all() and (pos[b, :, L:] == -3).all()
        assert (pos[b, :, L - n[b]:L] == b * 1000 + np.arange(n[b])).all()


def test_rows_that_are_no_nodes_add_nothing(torch):
    from paper_2510_26577_amd import evict
    rng = np.random.default_rng(4)
    lay = cc.Layout(rng, [50], 2, 128)
    four = cc.FourBit(rng, lay, [50])
    q, lse = cc.dev(orc.to_bf16(rng.standard_normal((6, 8, 128)))), cc.dev(np.full((6, 8), 4.0, np.float32))
    out = []
    for path in ([1, 9, 3], [1, -1, 3]):
        w = torch.ones((1, 2, 50), device="cuda")
        evict.key_weights(q=q, lse=lse, cache=four.cache, cu_T=cc.dev([0, 6], np.int32), L=cc.dev([50], np.int32), weight=w, max_rows=3, max_L=50,
                          scale=0.1, path=cc.dev([path], np.int32), path_len=cc.dev([3], np.int32))
        out.append(w.cpu().numpy())
    K = four.values(0, np.arange(50))[0]
    minus = np.array([4.0, -np.inf, 4.0])[:, None].repeat(8, 1)
    ref, off = orc.key_weights(np.ones((2, 50)), orc.bf16(cc.bits(q))[[1, 1, 3]], minus, K, 3, 0.1)
    assert np.array_equal(out[0], out[1]) and (np.abs(out[0][0] - ref) <= 2.0 ** -20 * off + 2.0 ** -20 * ref).all()


def test_key_weights_are_the_same_from_call_to_call_and_in_a_graph(torch):
    from paper_2510_26577_amd import evict
    rng = np.random.default_rng(14)
    lay = cc.Layout(rng, [900], 8, 128, 16)
    four = cc.FourBit(rng, lay, [900])
    q, lse = cc.dev(orc.to_bf16(rng.standard_normal((20, 32, 128)))), cc.dev(np.full((20, 32), 6.0, np.float32))
    w = torch.zeros((1, 8, 900), device="cuda")
    args = evict.make_key_weight_args(q=q, lse=lse, cache=four.cache, cu_T=cc.dev([0, 20], np.int32), L=cc.dev([900], np.int32), weight=w, max_rows=20,
                                      max_L=900, scale=0.1)
    eager = []
    for _ in range(4):
        evict.key_weights_raw(args)
        eager.append(w.clone())
    stream = torch.cuda.Stream()
    w.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        evict.key_weights_raw(args)
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, want)


# ---- the choice ----
def _weights(rng, shape, kind):
    if kind == "ties":
        return rng.integers(0, 4, shape).astype(np.float32)
    if kind == "equal":
        return np.full(shape, 0.25, np.float32)
    w = np.exp(rng.standard_normal(shape) * 3).astype(np.float32)
    w[rng.random(shape) < 0.2] = 0
    if kind == "odd":
        for x in (np.nan, -0.0, np.inf, -np.inf, -1.5, 1e-42):
            w[rng.random(shape) < 0.05] = x
    return w


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd"])
@pytest.mark.parametrize("lengths,keep", [([1, 2, 3], [1, 1, 0]), ([64, 65, 63, 0], [32, 64, 62, 5]), ([1000, 700, 1024], [500, 1, 1023]),
                                          ([1025, 4096, 4097], [1024, 64, 4000]), ([5000, 100], [2500, 200])])
def test_choice_of_slots(torch, lengths, keep, kind):
    from paper_2510_26577_amd import evict
    say(f"[case] choice lengths={lengths} keep={keep} {kind}")
    rng = np.random.default_rng(len(lengths) + lengths[0])
    B, H, layers, ld = len(lengths), 2, 2, max(lengths) + 3
    w = _weights(rng, (layers, B, H, ld), kind)
    pos = rng.permuted(np.broadcast_to(np.arange(ld, dtype=np.int32), w.shape), axis=-1)
    newest = np.array([L - L // 5 for L in lengths], np.int32)
    dw, dp, dl, dk, dn = cc.dev(w), cc.dev(pos), cc.dev(lengths, np.int32), cc.dev(keep, np.int32), cc.dev(newest)
    for n_first, new, ages in ((0, None, None), (3, None, None), (0, newest, None), (2, newest, pos), (10 ** 6, None, None)):
        src = torch.full((layers, B, H, max(keep) + 1), -9, dtype=torch.int32, device="cuda")
        got, L_out = evict.select(dw, dl, dk, max_L=max(lengths), max_keep=0, n_first=n_first, newest=None if new is None else dn,
                                  pos=None if ages is None else dp, src=src)
        got = got.cpu().numpy()
        assert L_out.tolist() == [max(0, min(k, L)) for k, L in zip(keep, lengths)]
        for layer in range(layers):
            for b in range(B):
                for h in range(H):
                    ref = orc.select(w[layer, b, h, :lengths[b]], keep[b], n_first, None if new is None else new[b],
                                     None if ages is None else ages[layer, b, h, :lengths[b]])
                    assert np.array_equal(got[layer, b, h, :len(ref)], ref) and (got[layer, b, h, len(ref):] == -9).all()


@pytest.mark.parametrize("L,keep", [(32768, 16000), (32769, 32000), (200000, 150001), (262144, 1000)])
def test_choice_among_many_slots(torch, L, keep):
    from paper_2510_26577_amd import evict
    say(f"[case] choice L={L} keep={keep}")
    rng = np.random.default_rng(L)
    w = _weights(rng, (1, 2, L), "ties" if keep == 1000 else "plain")
    src, n = evict.select(cc.dev(w), cc.dev([L], np.int32), cc.dev([keep], np.int32), max_L=L, max_keep=keep, n_first=4, newest=cc.dev([L - 500], np.int32))
    for h in range(2):
        assert np.array_equal(src[0, h].cpu().numpy(), orc.select(w[0, h], keep, 4, L - 500))


def test_longer_sequences_end_at_the_bound_and_no_row_keeps_more_than_it_has_room_for(torch):
    from paper_2510_26577_amd import evict
    w = cc.dev(np.arange(200, dtype=np.float32)[None, None])
    src, n = evict.select(w, cc.dev([200], np.int32), cc.dev([10], np.int32), max_L=100, max_keep=10)
    assert src[0, 0].tolist() == list(range(90, 100)) and n.tolist() == [10]
    src, n = evict.select(w, cc.dev([200], np.int32), cc.dev([-5], np.int32), max_L=200, max_keep=10)
    assert n.tolist() == [0]
    src, n = evict.select(w, cc.dev([200], np.int32), cc.dev([150], np.int32), max_L=200, max_keep=10)
    assert src[0, 0].tolist() == list(range(190, 200)) and n.tolist() == [10]


# ---- the move ----
@pytest.mark.parametrize("rows,D", [("bf16", 128), ("bf16", 64), ("e4m3", 128), ("e4m3", 64), ("e2m1", 128), ("e2m1", 64)])
@pytest.mark.parametrize("page,head_major,shared,layers", [(0, False, False, 2), (16, True, False, 1), (0, True, True, 2), (7, False, True, 1)])
def test_rows_move_into_the_gaps(torch, rows, D, page, head_major, shared, layers):
    from paper_2510_26577_amd import cache4, evict
    say(f"[case] move rows={rows} D={D} page={page} shared={shared}")
    rng = np.random.default_rng(D + page)
    Hkv, lengths, keep = 3, [200, 65, 64, 1], [100, 64, 80, 1]
    H, B, ld = 1 if shared else Hkv, 4, 210
    lay = cc.Layout(rng, lengths, Hkv, D, page, head_major)
    if rows == "e2m1":
        four = cc.FourBit(rng, lay, lengths, layers)
        cache, host, dev = four.cache, [four.k, four.ks, four.v, four.vs], [four.d[x] for x in ("k", "k_row_scale", "v", "v_row_scale")]
    else:
        kind = {"bf16": np.uint16, "e4m3": np.uint8}[rows]
        host = [rng.integers(0, 256 if rows == "e4m3" else 65536, (lay.rows * layers, D)).astype(kind) for _ in range(2)]
        dev = [cc.dev(x) for x in host]
        cache = lay.cache(kind=cache4.ROWS_BF16 if rows == "bf16" else cache4.ROWS_E4M3, k=dev[0], v=dev[1])
    w, pos = rng.random((layers, B, H, ld)).astype(np.float32), rng.integers(0, 1000, (layers, B, H, ld)).astype(np.int32)
    dw, dp = cc.dev(w), cc.dev(pos)
    src, n = evict.select(dw, cc.dev(lengths, np.int32), cc.dev(keep, np.int32), max_L=max(lengths), max_keep=max(keep))
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    evict.move(src=src, n=n, cache=cache, Hkv=Hkv, D=D, max_keep=max(keep), weight=dw, pos=dp, layer_stride_cache=lay.rows * D, err_flag=flag)
    torch.cuda.synchronize()
    s, want, ww, wp = src.cpu().numpy(), [x.copy() for x in host], w.copy(), pos.copy()
    for layer in range(layers):
        for b in range(B):
            k = min(keep[b], lengths[b])
            for h in range(Hkv):
                old = s[layer, b, 0 if shared else h, :k]
                for x, y in zip(want, host):
                    x[lay.at(b, np.arange(k))[:, h] + layer * lay.rows] = y[lay.at(b, old)[:, h] + layer * lay.rows]
            for h in range(H):
                ww[layer, b, h, :k], wp[layer, b, h, :k] = w[layer, b, h, s[layer, b, h, :k]], pos[layer, b, h, s[layer, b, h, :k]]
    assert not flag.item() and np.array_equal(dw.cpu().numpy(), ww) and np.array_equal(dp.cpu().numpy(), wp)
    for x, y in zip(dev, want):
        assert np.array_equal(cc.bits(x) if x.dtype == torch.bfloat16 else x.cpu().numpy(), y)


def test_entries_that_are_no_moves_are_left_out(torch):
    from paper_2510_26577_amd import cache4, evict
    rng = np.random.default_rng(3)
    lay = cc.Layout(rng, [40, 40], 2, 128, 16)  # (room: 48)
    for b, j, old, bad in ((0, 3, 30, 0), (1, 3, 2, 2), (0, 3, 48, 1), (1, 0, -1, 2), (0, 5, 1 << 30, 1), (0, 5, 45, 1)):
        x = orc.to_bf16(rng.standard_normal((lay.rows, 128)))
        d = cc.dev(x)
        src = np.tile(np.arange(20, dtype=np.int32), (2, 2, 1))
        src[b, 1, j] = old
        w = torch.rand((2, 2, 40), device="cuda")
        w0, flag = w.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        evict.move(src=cc.dev(src), n=cc.dev([20, 20], np.int32), cache=lay.cache(kind=cache4.ROWS_BF16, k=d, v=d.clone()), Hkv=2, D=128, max_keep=20,
                   weight=w, err_flag=flag)
        assert flag.item() == bad
        if bad:
            assert np.array_equal(cc.bits(d), x) and torch.equal(w, w0)
        else:
            x[lay.at(b, [j])[0, 1]] = x[lay.at(b, [old])[0, 1]]
            w0[b, 1, j] = w0[b, 1, old]
            assert np.array_equal(cc.bits(d), x) and torch.equal(w, w0)


# ---- together ----
def test_a_step_in_a_graph_and_on_another_stream(torch):
    """Commit, weights, choice and move captured once: every replay gives what the eager calls give, on a stream of their own too."""
    from paper_2510_26577_amd import cache4, evict
    rng = np.random.default_rng(31)
    Hq, Hkv, D, layers, T, L0 = 8, 2, 128, 2, 10, [60, 150]
    lay = cc.Layout(rng, [160, 160], Hkv, D, 16)
    four = cc.FourBit(rng, lay, L0, layers)
    k, v = (cc.dev(orc.to_bf16(rng.standard_normal((layers, 2 * T, Hkv, D)))) for _ in range(2))
    q, lse = cc.dev(orc.to_bf16(rng.standard_normal((2 * T, Hq, D)))), cc.dev(np.full((2 * T, Hq), 5.0, np.float32))
    cu_T, L, keep = cc.dev([0, T, 2 * T], np.int32), cc.dev(L0, np.int32), cc.dev([50, 100], np.int32)
    path, n = cc.dev([[0, 3, 7], [0, 1, -1]], np.int32), cc.dev([3, 2], np.int32)
    weight, pos = cc.dev(rng.random((layers, 2, Hkv, 160)).astype(np.float32)), torch.zeros((layers, 2, Hkv, 160), dtype=torch.int32, device="cuda")
    L_new, L_kept, flag = (torch.zeros(m, dtype=torch.int32, device="cuda") for m in (2, 2, 1))
    src = torch.zeros((layers, 2, Hkv, 100), dtype=torch.int32, device="cuda")
    store = cache4.make_rows_args(k_rows=k, v_rows=v, cu_T=cu_T, L=L, cache=four.cache, max_rows=3, path=path, path_len=n, L_out=L_new, err_flag=flag,
                                  n_layers=layers, layer_stride_cache=lay.rows * D, layer_stride_rows=2 * T * Hkv * D)
    weigh = [evict.make_key_weight_args(q=q, lse=lse, cache=lay.cache(**{x: t[i * lay.rows:(i + 1) * lay.rows] for x, t in four.d.items()}), cu_T=cu_T,
                                        L=L_new, weight=weight[i], pos=pos[i], first_pos=L, max_rows=3, max_L=160, scale=0.1, path=path, path_len=n)
             for i in range(layers)]
    choose = evict.make_select_args(weight=weight, L=L_new, keep=keep, max_L=160, src=src, L_out=L_kept, n_first=2, newest=L, pos=pos)
    shift = evict.make_move_args(src=src, n=L_kept, cache=four.cache, Hkv=Hkv, D=D, max_keep=100, weight=weight, pos=pos,
                                 layer_stride_cache=lay.rows * D, err_flag=flag)
    state = [*four.d.values(), weight, pos, src, L_new, L_kept]
    first = [t.clone() for t in state]

    def reset():
        for t, x in zip(state, first):
            t.copy_(x)

    def step(stream=None):
        cache4.store_raw(store, stream)
        for a in weigh:
            evict.key_weights_raw(a, stream)
        evict.select_raw(choose, stream)
        evict.move_raw(shift, stream)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in state]
    assert L_kept.tolist() == [50, 100] and not flag.item() and not torch.equal(want[0], first[0])
    same = lambda: all(torch.equal(t.view(torch.uint8), x.view(torch.uint8)) for t, x in zip(state, want))
    other = torch.cuda.Stream()
    reset()
    torch.cuda.synchronize()
    step(other)
    other.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        step()
    for _ in range(4):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        reset()
        step()
        torch.cuda.synchronize()
        assert same()


def test_a_cache_over_its_budget(torch):
    """Prompts stored, then steps of attention, acceptance, commit and weighing; whenever a sequence is over the budget its slots are
    chosen and moved.  Every step's attention is compared with 64 bits on the values the cache should hold."""
    from paper_2510_26577_amd import cache4, evict, verify
    rng = np.random.default_rng(21)
    Hq, Hkv, D, B, page, budget, steps, T = 8, 2, 128, 2, 16, 90, 12, 12
    scale = 1.0 / np.sqrt(D)
    prompts, room = [80, 37], 112
    lay = cc.Layout(rng, [room] * B, Hkv, D, page)
    cache = cc.FourBit(rng, lay, [0] * B)
    cu = np.concatenate([[0], np.cumsum(prompts)]).astype(np.int32)
    k, v = (orc.to_bf16(rng.standard_normal((sum(prompts), Hkv, D))) for _ in range(2))
    L = torch.zeros(B, dtype=torch.int32, device="cuda")
    n = torch.zeros(B, dtype=torch.int32, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache4.store(k_rows=cc.dev(k), v_rows=cc.dev(v), cu_T=cc.dev(cu), L=L, cache=cache.cache, max_rows=max(prompts), L_out=n, err_flag=flag)
    L, n = n, L
    weight, pos = torch.zeros((B, Hkv, room), device="cuda"), torch.zeros((B, Hkv, room), dtype=torch.int32, device="cuda")
    pos[:] = torch.arange(room, dtype=torch.int32, device="cuda")
    total = list(prompts)  # tokens so far
    # what the cache should hold: per sequence and head, values by slot
    def rounded(x, which):
        e = orc.encode_rows(x, x)
        return orc.decode_k(*e[:2]) if which == "k" else orc.decode_v(*e[2:])
    K = [rounded(k[cu[b]:cu[b + 1]], "k") for b in range(B)]
    V = [rounded(v[cu[b]:cu[b + 1]], "v") for b in range(B)]
    W = [np.zeros((Hkv, p)) for p in prompts]
    evictions = 0
    for step in range(steps):
        parents = cc.trees(rng, [T] * B, 5)
        cu_T = cc.dev(np.arange(B + 1) * T, np.int32)
        q, kt, vt = (orc.to_bf16(rng.standard_normal((B * T, h, D))) for h in (Hq, Hkv, Hkv))
        draft = rng.integers(0, 100, B * T).astype(np.int32)
        target = rng.integers(0, 100, B * T).astype(np.int32)
        for b in range(B):
            for i in range(T):
                kids = np.nonzero(parents[b] == i)[0]
                if len(kids):
                    target[b * T + i] = draft[b * T + int(kids[0])]
        d = [cc.dev(x) for x in (q, kt, vt)]
        parent = cc.dev(np.concatenate(parents))
        out, lse = cache4.tree_verify_attn(*d, cache.cache, cu_T, L, max_T=T, max_L=room, scale=scale, parent=parent)
        path, path_len, _ = verify.accept_greedy(parent, cu_T, cc.dev(draft), cc.dev(target), 6)
        cache4.store(k_rows=d[1], v_rows=d[2], cu_T=cu_T, L=L, cache=cache.cache, max_rows=6, path=path, path_len=path_len, L_out=n, err_flag=flag)
        L, n = n, L
        evict.key_weights(q=d[0], lse=lse, cache=cache.cache, cu_T=cu_T, L=L, weight=weight, max_rows=6, max_L=room, scale=scale, path=path,
                          path_len=path_len, pos=pos, first_pos=cc.dev(total, np.int32))
        got, got_lse = orc.bf16(cc.bits(out)), lse.double().cpu().numpy()
        paths, lens = path.cpu().numpy(), path_len.tolist()
        for b in range(B):
            r = slice(b * T, (b + 1) * T)
            see = np.concatenate([np.ones((T, len(K[b])), bool), cc.ancestor_sets(parents[b])], 1)
            ref = orc.attention(orc.bf16(q[r]), np.concatenate([K[b], orc.bf16(kt[r])]), np.concatenate([V[b], orc.bf16(vt[r])]), see, scale)
            compare(got[r], got_lse[r], *ref)
            nodes = b * T + paths[b, :lens[b]]
            K[b], V[b] = np.concatenate([K[b], rounded(kt[nodes], "k")]), np.concatenate([V[b], rounded(vt[nodes], "v")])
            W[b], off = orc.key_weights(np.concatenate([W[b], np.zeros((Hkv, lens[b]))], 1), orc.bf16(q[nodes]), got_lse[nodes], K[b], lens[b], scale)
            assert np.abs(weight[b, :, :len(K[b])].cpu().numpy() - W[b]).max() <= (step + 1) * (2.0 ** -20 * off.max() + 2.0 ** -20 * (W[b].max() + 1))
            total[b] += lens[b]
        lengths = L.tolist()
        assert lengths == [len(x) for x in K] and not flag.item()
        if max(lengths) > budget:
            evictions += 1
            keep = cc.dev([70, 200], np.int32)
            src, n = evict.select(weight, L, keep, max_L=room, max_keep=room, n_first=4, newest=cc.dev([t - 10 for t in total], np.int32), pos=pos)
            w, p, s = weight.cpu().numpy(), pos.cpu().numpy(), src.cpu().numpy()
            evict.move(src=src, n=n, cache=cache.cache, Hkv=Hkv, D=D, max_keep=room, weight=weight, pos=pos, err_flag=flag)
            for b in range(B):
                m = min([70, 200][b], lengths[b])
                for g in range(Hkv):
                    ref = orc.select(w[b, g, :lengths[b]], m, 4, total[b] - 10, p[b, g, :lengths[b]])
                    assert np.array_equal(s[b, g, :m], ref)
                    K[b][:m, g], V[b][:m, g], W[b][g, :m] = K[b][ref, g], V[b][ref, g], W[b][g, ref]
                K[b], V[b], W[b] = K[b][:m], V[b][:m], W[b][:, :m]
            L = n
            n = torch.zeros(B, dtype=torch.int32, device="cuda")
            assert L.tolist() == [len(x) for x in K] and not flag.item()
            for b in range(B):  # the ten newest tokens are still there
                for g in range(Hkv):
                    ages = set(pos[b, g, :len(K[b])].tolist())
                    assert set(range(total[b] - 10, total[b])) <= ages
    assert evictions >= 2
