"""GPU tests of tva_chunk_attn: windows with both head dimensions in every size of a workgroup, and the precision that each size has in whole steps."""
import numpy as np
import pytest

from oracle import cache_oracle, layer_oracle as orc
from tests import cache_cases as cc
from tests.test_gpu_chunk import _attend, compare

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
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,head_major", [(0, False), (16, True), (24, False), (5, False)])
@pytest.mark.parametrize("window,n_first", [(1, 0), (33, 4), (64, 65), (200, 1), (1000, 130)])
def test_windows_with_both_head_dimensions(torch, rows, plan, D, page, head_major, window, n_first):
    _attend(torch, np.random.default_rng(window + page), (8, 2, D), [130, 1, 40, 5], [500, 700, 0, 66], page, head_major, rows=rows, window=window, n_first=n_first, plan=plan,
            splits=window % 2 * 3)


@pytest.mark.parametrize("plan", [32, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_the_weights_of_a_step_have_the_digits_of_their_workgroup(torch, plan, D, tree):
    """append, then the attention of what was appended: a weight has 16 bits in 32-row workgroups, 8 in the others."""
    from paper_2510_26577_amd import chunk, rotary
    Hq, Hkv, B = 8, 2, 2
    rng = np.random.default_rng(plan + D)
    sizes, lengths = [60, 7], [300, 41]
    n, total = sum(sizes), [a + b for a, b in zip(sizes, lengths)]
    lay = cc.Layout(rng, total, Hkv, D, 16)
    dk, dv = (cc.dev(to_bf16(rng.standard_normal((lay.rows, D)))) for _ in range(2))
    cache = lay.cache(kind=0, k=dk, v=dv)
    sets = [cc.ancestor_sets(p) for p in cc.trees(rng, sizes)] if tree else [None] * B
    mask = cc.dev(np.concatenate([cc.mask_words(s, 1) for s in sets])) if tree else None
    x, cu, L = cc.dev(to_bf16(rng.standard_normal((n, Hq + 2 * Hkv, D)))), cc.dev(np.concatenate([[0], np.cumsum(sizes)]), np.int32), cc.dev(lengths, np.int32)
    q = rotary.append(q=x[:, :Hq], k=x[:, Hq:Hq + Hkv], v=x[:, Hq + Hkv:], cache=cache, cu_T=cu, L=L, freq=cc.dev(rotary.frequencies(D)[0]), dims=D, anc_mask=mask)
    out, lse = torch.zeros((n, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, Hq), device="cuda")
    args = chunk.make_args(q=q, cache=cache, cu_T=cu, L=L, Hkv=Hkv, max_T=max(sizes), max_L=max(lengths), scale=D ** -0.5, anc_mask=mask, out=out, lse=lse, plan_rows=plan)
    chunk.attn_workspace(args, "cuda")
    chunk.attn_raw(args)
    torch.cuda.synchronize()
    K, V, got, got_lse, held = bf16(cc.bits(dk)), bf16(cc.bits(dv)), bf16(cc.bits(out)), lse.double().cpu().numpy(), bf16(cc.bits(q))
    for b in range(B):
        r, at = slice(sum(sizes[:b]), sum(sizes[:b + 1])), lay.at(b, np.arange(total[b]))
        ok, _ = orc.seen(lengths[b], sizes[b], sets=sets[b])
        ro, rl, size, reach = orc.attention(held[r], K[at], V[at], ok, D ** -0.5)
        compare(got[r], got_lse[r], ro, rl, size, reach, 2.0 ** -16 if chunk.plan_rows(args) == 32 else 2.0 ** -8)
