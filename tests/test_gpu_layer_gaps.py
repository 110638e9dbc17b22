"""GPU tests of tva_chunk_attn over page tables with entries below 0, the cache in the middle of larger tensors."""
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


@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
@pytest.mark.parametrize("plan", [32, 128, 256])
@pytest.mark.parametrize("page", [4, 5, 16, 24])
@pytest.mark.parametrize("D,tree", [(64, False), (128, False), (128, True)])
def test_pages_that_are_gone_beside_values_that_are_not_finite(torch, rows, plan, page, D, tree):
    """Entries of -1 where no token sees a position of the page, in tiles that are marked: page 0, read in their place, holds NaN, a value that is
    seen is infinite, and what lies in front of the cache and behind it (eight pages of each) is NaN and stays as it is."""
    from paper_2510_26577_amd import cache4, chunk
    Hq, Hkv, B, spare = 8, 2, 2, 8
    sizes, lengths, window, first = [9, 40], [517, 301], 130, 3
    rng = np.random.default_rng(1000 * page + plan)
    total = [L + T for L, T in zip(lengths, sizes)]
    n = [-(-x // page) for x in total]
    table, at = np.full((B, max(n) + 1), -1, np.int32), 0
    pool = 1 + rng.permutation(sum(n)).astype(np.int32)
    for b in range(B):
        table[b, :n[b]] = pool[at:at + n[b]]
        at += n[b]
    shape = ((sum(n) + 1 + 2 * spare) * page, Hkv, D)
    if rows == "bf16":
        k, v = (to_bf16(rng.standard_normal(shape)) for _ in range(2))
        nan, inf, more, value = 0x7FC0, 0x7F80, {}, lambda x, _: bf16(x)
    else:
        k, v = (rng.integers(0, 0x60, shape).astype(np.uint8) + 128 * rng.integers(0, 2, shape).astype(np.uint8) for _ in range(2))
        nan, inf, more = 0x7F, 0xFF, dict(k_scale=0.125, v_scale=0.25)
        value = lambda x, name: fp8_oracle.e4m3_decode(x) * more[name]  # noqa: E731
    inside = slice(spare * page, -spare * page)
    for x in (k, v):
        x[:(spare + 1) * page] = x[-spare * page:] = nan
    sets = [cc.ancestor_sets(p) for p in cc.trees(rng, sizes)] if tree else [None] * B
    seen = [orc.seen(L, T, window, first, s)[0] for L, T, s in zip(lengths, sizes, sets)]
    place = [table[b, np.arange(total[b]) // page] * page + np.arange(total[b]) % page for b in range(B)]
    for b in range(B):
        v[spare * page + place[b][lengths[b] - window + 4], 1, 7] = inf  # at the window's edge: some rows see it, or all
        v[spare * page + place[b][1], 0, 9] = inf                         # among the first tokens
    gone = 0
    for b in range(B):
        for i in range(n[b]):
            if not seen[b][:, i * page:(i + 1) * page].any():
                table[b, i] = -1
                gone += page
    assert gone > 300
    q = to_bf16(rng.standard_normal((sum(sizes), Hq, D)))
    dk, dv = cc.dev(k), cc.dev(v)
    before = dk.clone(), dv.clone()
    cache = cache4.make_cache(kind=["bf16", "e4m3"].index(rows), k=dk[inside], v=dv[inside], page_table=cc.dev(table), page_size=page, **more)
    out, lse = torch.zeros((sum(sizes), Hq, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((sum(sizes), Hq), device="cuda")
    args = chunk.make_args(q=cc.dev(q), cache=cache, cu_T=cc.dev(np.concatenate([[0], np.cumsum(sizes)]), np.int32), L=cc.dev(lengths, np.int32), Hkv=Hkv, max_T=max(sizes),
                           max_L=max(lengths), scale=D ** -0.5, window=window, n_first=first, plan_rows=plan, out=out, lse=lse,
                           anc_mask=cc.dev(np.concatenate([cc.mask_words(s, 1) for s in sets])) if tree else None)
    chunk.attn_workspace(args, "cuda")
    chunk.attn_raw(args)
    torch.cuda.synchronize()
    for t, was in zip((dk, dv), before):
        assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))
    got, got_lse, step = bf16(cc.bits(out)), lse.double().cpu().numpy(), 2.0 ** -16 if plan == 32 else 2.0 ** -8
    for b in range(B):
        r = slice(sum(sizes[:b]), sum(sizes[:b + 1]))
        K, V = value(k[inside][place[b]], "k_scale"), value(v[inside][place[b]], "v_scale")
        ro, rl, size, reach = orc.attention(bf16(q[r]), K, V, seen[b], D ** -0.5)
        assert not np.isfinite(ro).all()
        compare(got[r], got_lse[r], ro, rl, size, reach, step)
