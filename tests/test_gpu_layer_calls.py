"""GPU tests of the operators of include/tva_layer.h as a program uses them: together, in graphs, on other streams, far into large caches."""
import numpy as np
import pytest

from oracle import cache_oracle, fp8_oracle, layer_oracle as orc
from tests import cache_cases as cc
from tests.test_gpu_chunk import compare

pytestmark = pytest.mark.gpu
bf16, to_bf16 = cache_oracle.bf16, cache_oracle.to_bf16


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def same(a, b):
    import torch
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


class Layer:
    """One layer of a model with norms of its heads and a window: projections of tokens in, attention out, its cache kept in pages."""

    def __init__(self, torch, rows, window, B=2, heads=(8, 2, 64), room=600, page=16):
        from paper_2510_26577_amd import rotary
        self.torch, self.rows, self.window, self.first, self.B, self.heads = torch, rows, window, 4 if window else 0, B, heads
        Hq, Hkv, D = heads
        rng = np.random.default_rng(7)
        self.lay = cc.Layout(rng, [room] * B, Hkv, D, page)
        self.scales = dict(k_scale=0.02, v_scale=0.015) if rows == "e4m3" else {}
        self.k, self.v = (torch.zeros((self.lay.rows, D), dtype=torch.bfloat16 if rows == "bf16" else torch.uint8, device="cuda") for _ in range(2))
        self.cache = self.lay.cache(kind=0 if rows == "bf16" else 1, k=self.k, v=self.v, **self.scales)
        self.freq, self.magnitude = rotary.frequencies(48, scaling=rotary.RAMP, factor=4.0, original=512.0)
        self.norms = [to_bf16(1 + 0.2 * rng.standard_normal(D)) for _ in range(2)]
        self.d = [cc.dev(x) for x in (self.freq, *self.norms)]
        self.L = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.host_L, self.past = [0] * B, [[np.zeros((0, h, D)) for h in (Hkv, Hkv)] for _ in range(B)]

    def step(self, rng, sizes, tree=False, stream=None, keep=True):
        """The library's step and the definition's; what is cached (rounded as the cache holds it) is compared on the way."""
        from paper_2510_26577_amd import chunk, rotary
        Hq, Hkv, D = self.heads
        cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        n = int(cu[-1])
        x = to_bf16(rng.standard_normal((n, Hq + 2 * Hkv, D)))
        dx, dcu = cc.dev(x), cc.dev(cu)
        sets = [cc.ancestor_sets(p) for p in cc.trees(rng, sizes)] if tree else None
        mask = cc.dev(np.concatenate([cc.mask_words(s, 1) for s in sets])) if tree else None
        self.torch.cuda.synchronize()
        L_out = self.torch.zeros_like(self.L)
        q = rotary.append(q=dx[:, :Hq], k=dx[:, Hq:Hq + Hkv], v=dx[:, Hq + Hkv:], cache=self.cache, cu_T=dcu, L=self.L, anc_mask=mask, freq=self.d[0], dims=48,
                          magnitude=self.magnitude, q_norm=self.d[1], k_norm=self.d[2], eps=1e-6, L_out=L_out, stream=stream)
        out, lse = chunk.attn(q, self.cache, dcu, self.L, Hkv=Hkv, max_T=max(sizes), max_L=max(self.host_L), scale=D ** -0.5, window=self.window,
                              n_first=self.first, anc_mask=mask, stream=stream)
        self.torch.cuda.synchronize()
        got, got_lse, held = bf16(cc.bits(out)), lse.double().cpu().numpy(), (self.k.cpu(), self.v.cpu())
        for b, T in enumerate(sizes):
            r, L = slice(cu[b], cu[b + 1]), self.host_L[b]
            ok, pos = orc.seen(L, T, self.window, self.first, None if sets is None else sets[b])
            rq, _ = orc.heads(bf16(x[r, :Hq]), pos, self.freq, 48, False, self.magnitude, bf16(self.norms[0]), 1e-6)
            rk, _ = orc.heads(bf16(x[r, Hq:Hq + Hkv]), pos, self.freq, 48, False, self.magnitude, bf16(self.norms[1]), 1e-6)
            at = self.lay.at(b, L + np.arange(T))
            if self.rows == "bf16":
                k, v = (bf16(cc.bits(h[self.torch.from_numpy(at)])) for h in held)
            else:
                k, v = (fp8_oracle.e4m3_decode(h.numpy()[at]) * s for h, s in zip(held, self.scales.values()))
            # stored keys: half a step of bf16, and of the 8-bit code (2^-4 of the value, 2^-10 of the scale among the smallest)
            off = 2.0 ** -8 * 1.01 * np.abs(rk) + 2.0 ** -17
            if self.rows == "e4m3":
                off += 2.0 ** -4 * (np.abs(rk) + off) + 2.0 ** -10 * self.scales["k_scale"]
            assert (np.abs(np.clip(rk, -448 * self.scales.get("k_scale", 1), 448 * self.scales.get("k_scale", 1)) - k) <= off).all()
            K, V = np.concatenate([self.past[b][0], k]), np.concatenate([self.past[b][1], v])
            # the attention, of q as it was rounded: what reads it is checked to the attention's own tolerance
            q_held = bf16(cc.bits(q[r]))
            assert (np.abs(q_held - rq) <= 2.0 ** -8 * 1.01 * np.abs(rq) + 2.0 ** -17).all()
            ro, rl, size, reach = orc.attention(q_held, K, V, ok, D ** -0.5)
            compare(got[r], got_lse[r], ro, rl, size, reach, 2.0 ** -8)
            if keep:
                self.past[b], self.host_L[b] = [K, V], L + T
        assert L_out.tolist() == [L + T for L, T in zip(self.host_L, [0] * len(sizes) if keep else sizes)]
        if keep:
            self.L.copy_(L_out)


@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
@pytest.mark.parametrize("window", [0, 90])
def test_prompts_in_chunks_then_tokens_then_trees(torch, rows, window):
    layer, rng = Layer(torch, rows, window), np.random.default_rng(1)
    layer.step(rng, [150, 7])           # prompts' first chunks
    layer.step(rng, [90, 200])          # their next
    for _ in range(3):
        layer.step(rng, [1, 1])         # plain decoding
    layer.step(rng, [30, 9], tree=True, keep=False)  # a draft tree, of which nothing is kept
    layer.step(rng, [1, 3])
    layer.step(rng, [0, 2])


def test_a_step_on_another_stream(torch):
    layer, rng = Layer(torch, "bf16", 40), np.random.default_rng(2)
    s = torch.cuda.Stream()
    layer.step(rng, [300, 200], stream=s)
    layer.step(rng, [2, 1], stream=s)


def _blocks(torch, rng, T, L, splits=0, plan=0, out=None):
    """Argument blocks of one step over a paged cache: (append's, attention's, tensors)."""
    from paper_2510_26577_amd import chunk, rotary
    Hq, Hkv, D, B = 8, 2, 128, len(L)
    lay = cc.Layout(rng, [int(l) + T + 64 for l in L], Hkv, D, 16)
    k, v = (torch.randn((lay.rows, D), device="cuda").bfloat16() for _ in range(2))
    x, freq = torch.randn((B * T, Hq + 2 * Hkv, D), device="cuda").bfloat16(), cc.dev(rotary.frequencies(D)[0])
    cu, lengths = cc.dev(np.arange(B + 1) * T, np.int32), cc.dev(np.array(L, np.int32))
    cache = lay.cache(kind=0, k=k, v=v)
    q = torch.zeros((B * T, Hq, D), dtype=torch.bfloat16, device="cuda")
    a = rotary.make_append_args(q=x[:, :Hq], k=x[:, Hq:Hq + Hkv], v=x[:, Hq + Hkv:], q_out=q, cache=cache, cu_T=cu, L=lengths, freq=freq, dims=D)
    out, lse = torch.zeros_like(q), torch.zeros((B * T, Hq), device="cuda")
    c = chunk.make_args(q=q, cache=cache, cu_T=cu, L=lengths, Hkv=Hkv, max_T=T, max_L=max(L) + 32, scale=0.09, out=out, lse=lse, num_splits=splits, plan_rows=plan)
    chunk.attn_workspace(c, "cuda")
    return a, c, dict(x=x, q=q, k=k, v=v, out=out, lse=lse, L=lengths)


@pytest.mark.parametrize("T,L,splits", [(1, [700, 33, 5], 0), (1, [2000], 8), (40, [300, 90], 3), (7, [64, 0, 1000, 3], 1)])
def test_a_captured_step_replayed_with_other_lengths(torch, T, L, splits):
    """The graph reads lengths and rows where they are: replays between eager calls and synchronisations, each like the eager result."""
    from paper_2510_26577_amd import chunk, rotary
    rng = np.random.default_rng(3)
    a, c, t = _blocks(torch, rng, T, L, splits)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        rotary.append_raw(a)
        chunk.attn_raw(c)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            rotary.append_raw(a)
            chunk.attn_raw(c)
    for n in range(4):
        t["x"].copy_(torch.randn_like(t["x"]))
        t["L"].copy_(torch.tensor([max(0, l - n * 3) for l in L], dtype=torch.int32))
        rotary.append_raw(a)
        chunk.attn_raw(c)
        torch.cuda.synchronize()
        want = [t[x].clone() for x in ("out", "lse", "q", "k", "v")]
        for x in ("out", "lse", "q"):
            t[x].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(t[x], w) for x, w in zip(("out", "lse", "q", "k", "v"), want))


def test_graphs_that_share_a_workspace_one_after_the_other(torch):
    from paper_2510_26577_amd import chunk
    rng = np.random.default_rng(4)
    (_, c1, t1), (_, c2, t2) = _blocks(torch, rng, 2, [900], 6), _blocks(torch, rng, 33, [500, 40], 3)
    need = max(c1.workspace_bytes, c2.workspace_bytes)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    want = []
    for c, t in ((c1, t1), (c2, t2)):
        chunk.attn_raw(c)
        torch.cuda.synchronize()
        want.append(t["out"].clone())
        c.workspace, c.workspace_bytes = ws.data_ptr(), need
    s = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(s):
        for c in (c1, c2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                chunk.attn_raw(c)
            graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for i in order:
            (t1, t2)[i]["out"].zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        assert same(t1["out"], want[0]) and same(t2["out"], want[1])


def test_two_streams_at_once(torch):
    from paper_2510_26577_amd import chunk, rotary
    rng = np.random.default_rng(5)
    sets = [_blocks(torch, rng, 1, [3000], 16), _blocks(torch, rng, 300, [100, 900])]
    streams = [torch.cuda.Stream() for _ in sets]
    want = []
    for a, c, t in sets:
        rotary.append_raw(a)
        chunk.attn_raw(c)
        torch.cuda.synchronize()
        want.append((t["out"].clone(), t["lse"].clone()))
        t["out"].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for (a, c, t), s in zip(sets, streams):
            rotary.append_raw(a, s)
            chunk.attn_raw(c, s)
    torch.cuda.synchronize()
    assert all(same(t["out"], w[0]) and same(t["lse"], w[1]) for (_, _, t), w in zip(sets, want))


def test_results_do_not_change_from_call_to_call(torch):
    from paper_2510_26577_amd import chunk
    _, c, t = _blocks(torch, np.random.default_rng(6), 50, [4000, 700], 0)
    chunk.attn_raw(c)
    torch.cuda.synchronize()
    want = t["out"].clone(), t["lse"].clone()
    for _ in range(5):
        chunk.attn_raw(c)
    torch.cuda.synchronize()
    assert same(t["out"], want[0]) and same(t["lse"], want[1])


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
def test_places_beyond_32_bits_of_bytes_and_elements(torch, paged, rows):
    """Caches of more than 2^31 elements: the last pages, or the last rows of a dense cache."""
    from paper_2510_26577_amd import chunk, rotary
    Hq, Hkv, D, T, L = 8, 8, 128, 20, 70
    n = (1 << 31) // (Hkv * D) + 4096  # positions
    rng = np.random.default_rng(8)
    kind = torch.bfloat16 if rows == "bf16" else torch.uint8
    k, v = (torch.empty((n, Hkv, D), dtype=kind, device="cuda") for _ in range(2))
    if paged:
        table = np.array([[(n // 16) - 1, 0, (n // 16) - 3, 7, (n // 16) - 2, 11]], np.int32)
        at = (table[0, np.arange(L + T) // 16].astype(np.int64) * 16 + np.arange(L + T) % 16)
        place = dict(page_table=cc.dev(table), page_size=16)
    else:
        at = n - (L + T) - 5 + np.arange(L + T)
        place = dict(cu_L=cc.dev([n - (L + T) - 5, n - 5], np.int32))
    more = dict(k_scale=0.02, v_scale=0.02) if rows == "e4m3" else {}
    from paper_2510_26577_amd import cache4
    cache = cache4.make_cache(kind=0 if rows == "bf16" else 1, k=k, v=v, **place, **more)
    freq = cc.dev(rotary.frequencies(D)[0])
    x = to_bf16(rng.standard_normal((2, L + T, Hkv, D)))
    cu = lambda m: cc.dev([0, m], np.int32)  # noqa: E731
    zero, flag = cc.dev([0], np.int32), torch.zeros(1, dtype=torch.int32, device="cuda")
    rotary.append(k=cc.dev(x[0]), v=cc.dev(x[1]), cache=cache, cu_T=cu(L + T), L=zero, freq=freq, dims=D, err_flag=flag)
    q = to_bf16(rng.standard_normal((T, Hq, D)))
    out, lse = chunk.attn(cc.dev(q), cache, cu(T), cc.dev([L], np.int32), Hkv=Hkv, max_T=T, max_L=L, scale=D ** -0.5)
    torch.cuda.synchronize()
    assert int(flag) == 0
    held = [t[torch.from_numpy(at).cuda()].cpu() for t in (k, v)]
    if rows == "bf16":
        K, V = (bf16(cc.bits(h)) for h in held)
    else:
        K, V = (fp8_oracle.e4m3_decode(h.numpy()) * 0.02 for h in held)
    rk, _ = orc.heads(bf16(x[0]), np.arange(L + T), rotary.frequencies(D)[0], D)
    assert np.abs(K - rk).max() <= (2.0 ** -8 if rows == "bf16" else 2.0 ** -3.9) * np.abs(rk).max()
    ok, _ = orc.seen(L, T)
    ro, rl, size, reach = orc.attention(bf16(q), K, V, ok, D ** -0.5)
    compare(bf16(cc.bits(out)), lse.double().cpu().numpy(), ro, rl, size, reach, 2.0 ** -8)


def test_four_bit_prompts_are_read_by_the_attention_over_four_bit_rows(torch):
    """append to a cache of 4-bit rows, then the verification attention that reads them."""
    from paper_2510_26577_amd import cache4, rotary
    Hq, Hkv, D, L, T = 8, 2, 128, 100, 5
    rng = np.random.default_rng(9)
    lay = cc.Layout(rng, [L], Hkv, D, 16)
    held = dict(k=torch.zeros((lay.rows, D // 2), dtype=torch.uint8, device="cuda"), v=torch.zeros((lay.rows, D // 2), dtype=torch.uint8, device="cuda"),
                k_row_scale=torch.zeros((lay.rows, D // 32), dtype=torch.uint8, device="cuda"), v_row_scale=torch.zeros(lay.rows, dtype=torch.bfloat16, device="cuda"))
    cache = lay.cache(**held)
    freq = cc.dev(rotary.frequencies(D)[0])
    x = torch.randn((L, 2 * Hkv, D), device="cuda").bfloat16()
    k_out = torch.empty((L, Hkv, D), dtype=torch.bfloat16, device="cuda")
    rotary.append(k=x[:, :Hkv], v=x[:, Hkv:], k_out=k_out, cache=cache, cu_T=cc.dev([0, L], np.int32), L=cc.dev([0], np.int32), freq=freq, dims=D)
    q, kt, vt = (torch.randn((T, h, D), device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    parent = np.array([-1, 0, 0, 1, 3], np.int32)
    out, lse = cache4.tree_verify_attn(q, kt, vt, cache, cc.dev([0, T], np.int32), cc.dev([L], np.int32), max_T=T, max_L=L, scale=D ** -0.5, parent=cc.dev(parent))
    torch.cuda.synchronize()
    a, s, c, d = cache_oracle.encode_rows(cc.bits(k_out), cc.bits(x[:, Hkv:].contiguous()))
    K = np.concatenate([cache_oracle.decode_k(a, s), bf16(cc.bits(kt))])
    V = np.concatenate([cache_oracle.decode_v(c, d), bf16(cc.bits(vt))])
    seen = np.concatenate([np.ones((T, L), bool), cc.ancestor_sets(parent)], 1)
    ro, rl, size, reach = orc.attention(bf16(cc.bits(q)), K, V, seen, D ** -0.5)
    compare(bf16(cc.bits(out)), lse.double().cpu().numpy(), ro, rl, size, reach, 2.0 ** -8)


@pytest.mark.parametrize("rows", ["bf16", "e4m3", "e2m1"])
def test_entries_below_zero_are_no_pages(torch, rows):
    """Sequence 0 has two pages and the table's filling behind them: what would come after them is left out and flagged."""
    from paper_2510_26577_amd import cache4, rotary
    Hkv, D, page, kind = 2, 64, 16, ["bf16", "e4m3", "e2m1"].index(rows)
    table = np.array([[3, 1, -1, -1], [0, 4, 2, 5]], np.int32)
    width = D if kind < 2 else D // 2
    k, v = (torch.full((8 * page, Hkv, width), 3, dtype=torch.bfloat16 if kind == 0 else torch.uint8, device="cuda") for _ in range(2))
    more = dict(k_row_scale=torch.full((8 * page * Hkv, D // 32), 3, dtype=torch.uint8, device="cuda"),
                v_row_scale=torch.full((8 * page * Hkv,), 3, dtype=torch.bfloat16, device="cuda")) if kind == 2 else {}
    # (the cache handed over begins two pages into the memory, whose own pages 0 and 1 stay as they are)
    inner = dict(k=k[2 * page:], v=v[2 * page:], **{n: t[2 * page * Hkv:] for n, t in more.items()})
    cache = cache4.make_cache(kind=kind, page_table=cc.dev(table), page_size=page, **inner)
    x = torch.randn((30, 2 * Hkv, D), device="cuda").bfloat16()
    flag, L_out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    out = torch.zeros((30, Hkv, D), dtype=torch.bfloat16, device="cuda")
    rotary.append(k=x[:, :Hkv], v=x[:, Hkv:], k_out=out, cache=cache, cu_T=cc.dev([0, 20, 30], np.int32), L=cc.dev([20, 40], np.int32),
                  freq=cc.dev(rotary.frequencies(D)[0]), dims=D, L_out=L_out, err_flag=flag)
    torch.cuda.synchronize()
    assert int(flag) == 1 and L_out.tolist() == [40, 50] and bool((out != 0).any(2).all())
    at = np.concatenate([table[0, 1] * page + np.arange(4, 16), table[1, 2] * page + np.arange(8, 16), table[1, 3] * page + np.arange(2)]) + 2 * page
    wrote = (k != 3).any(2).any(1).cpu().numpy()
    assert sorted(np.nonzero(wrote)[0]) == sorted(at)
    assert bool((k[:2 * page] == 3).all()) and bool((v[:2 * page] == 3).all())


@pytest.mark.parametrize("plan", [32, 128, 256])
@pytest.mark.parametrize("page", [16, 4, 5])
def test_pages_that_the_window_has_left_may_be_gone(torch, page, plan):
    """Their entries are -1, and page 0, read in their place where a tile straddles the window's edge, holds NaN."""
    from paper_2510_26577_amd import cache4, chunk
    Hq, Hkv, D, T, L, window, first = 8, 2, 64, 9, 517, 130, 3
    rng = np.random.default_rng(10)
    pages = -(-(L + T) // page)
    table = 1 + rng.permutation(pages).astype(np.int32)[None]
    k, v = (rng.standard_normal(((pages + 1) * page, Hkv, D)) for _ in range(2))
    k[:page] = v[:page] = np.nan
    k, v, q = to_bf16(k), to_bf16(v), to_bf16(rng.standard_normal((T, Hq, D)))
    at = table[0, np.arange(L + T) // page] * page + np.arange(L + T) % page
    ok, _ = orc.seen(L, T, window, first)
    gone = [i for i in range(pages) if not ok[:, i * page:(i + 1) * page].any()]
    assert len(gone) * page > 300
    table[0, gone] = -1
    cache = cache4.make_cache(kind=0, k=cc.dev(k), v=cc.dev(v), page_table=cc.dev(table), page_size=page)
    out, lse = chunk.attn(cc.dev(q), cache, cc.dev([0, T], np.int32), cc.dev([L], np.int32), Hkv=Hkv, max_T=T, max_L=L, scale=D ** -0.5, window=window, n_first=first,
                          plan_rows=plan)
    torch.cuda.synchronize()
    ro, rl, size, reach = orc.attention(bf16(q), bf16(k[at]), bf16(v[at]), ok, D ** -0.5)
    compare(bf16(cc.bits(out)), lse.double().cpu().numpy(), ro, rl, size, reach, 2.0 ** -8)
