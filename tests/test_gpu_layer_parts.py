"""GPU tests of the operators of include/tva_layer.h on a part of a batch: cu_T does not begin at 0, the tensors are the whole batch's."""
import numpy as np
import pytest

from oracle import cache_oracle, layer_oracle as orc
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


@pytest.mark.parametrize("B,bound", [(1, 0), (1, 400), (5, 0), (64, 0), (65, 0), (70, 90)])
@pytest.mark.parametrize("plan", [32, 128, 256])
@pytest.mark.parametrize("tree", [False, True])
def test_the_later_sequences_of_a_batch(torch, B, bound, plan, tree):
    """bound: how much larger max_T is than it need be (one sequence is then found by its rows, as many are)."""
    if tree and bound > 64:
        bound = 64
    from paper_2510_26577_amd import chunk, rotary
    Hq, Hkv, D, skip = 8, 2, 64, 3
    rng = np.random.default_rng(10 * B + plan)
    sizes, lengths = rng.integers(0, 12, B + skip), rng.integers(0, 90, B + skip)
    sizes[:skip] = 170, 0, 131
    sizes[skip + B // 2] = 50
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n, begin = int(cu[-1]), int(cu[skip])
    lay = cc.Layout(rng, (lengths + sizes)[skip:].tolist(), Hkv, D, 16)
    k, v = (to_bf16(rng.standard_normal((lay.rows, D))) for _ in range(2))
    dk, dv = cc.dev(k), cc.dev(v)
    cache = lay.cache(kind=0, k=dk, v=dv)
    x = to_bf16(rng.standard_normal((n, Hq + 2 * Hkv, D)))
    dx, dcu, dL = cc.dev(x), cc.dev(cu)[skip:], cc.dev(lengths, np.int32)[skip:]
    freq, _ = rotary.frequencies(D)
    sets = [cc.ancestor_sets(p) for p in cc.trees(rng, sizes[skip:])] if tree else [None] * B
    mask = cc.dev(np.concatenate([np.full((begin, 2), 2 ** 64 - 1, np.uint64), *(cc.mask_words(s, 2) for s in sets)])) if tree else None
    q_out, k_out, out = (torch.full((n, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hq))
    lse, L_out, flag = torch.full((n, Hq), 7.0, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    rotary.append(q=dx[:, :Hq], k=dx[:, Hq:Hq + Hkv], v=dx[:, Hq + Hkv:], q_out=q_out, k_out=k_out, cache=cache, cu_T=dcu, L=dL, freq=cc.dev(freq), dims=D, anc_mask=mask,
                  L_out=L_out, err_flag=flag)
    chunk.attn(q_out, cache, dcu, dL, Hkv=Hkv, max_T=int(sizes[skip:].max()) + bound, max_L=int(lengths.max()), scale=D ** -0.5, anc_mask=mask, out=out, lse=lse, plan_rows=plan)
    torch.cuda.synchronize()
    assert all(bool((t[:begin] == 7).all()) for t in (q_out, k_out, out, lse))
    assert int(flag) == 0 and L_out.tolist() == (lengths + sizes)[skip:].tolist()
    held = [bf16(cc.bits(t)) for t in (dk, dv)]
    got, got_lse, got_q, got_k = bf16(cc.bits(out)), lse.double().cpu().numpy(), bf16(cc.bits(q_out)), bf16(cc.bits(k_out))
    mine = np.zeros(lay.rows, bool)
    for b in range(B):
        T, L, r = int(sizes[skip + b]), int(lengths[skip + b]), slice(cu[skip + b], cu[skip + b + 1])
        if T == 0:
            continue
        ok, pos = orc.seen(L, T, sets=sets[b])
        for have, cut in ((got_q, slice(0, Hq)), (got_k, slice(Hq, Hq + Hkv))):
            want, size = orc.heads(bf16(x[r, cut]), pos, freq, D)
            assert (np.abs(have[r] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size).all()
        at = lay.at(b, np.arange(L + T))
        mine[at[L:]] = True
        assert np.array_equal(held[0][at[L:]], got_k[r]) and np.array_equal(held[1][at[L:]], bf16(x[r, Hq + Hkv:]))
        ro, rl, size, reach = orc.attention(got_q[r], held[0][at], held[1][at], ok, D ** -0.5)
        compare(got[r], got_lse[r], ro, rl, size, reach, 2.0 ** -16 if plan == 32 else 2.0 ** -8)
    assert np.array_equal(held[0][~mine], bf16(k)[~mine]) and np.array_equal(held[1][~mine], bf16(v)[~mine])
