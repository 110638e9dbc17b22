"""Key weights (include/tva_cache.h) where rows are missing or keys are not finite."""
import numpy as np
import pytest

from oracle import cache_oracle as orc
from tests import cache_cases as cc
from tests.test_gpu_evict import torch  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def _close(got, ref, off, rows):
    """The bounds of test_gpu_evict.test_key_weights: 2^-20 of the exponentials' arguments, sums of `rows` terms in fp32."""
    tol = 2.0 ** -20 * off + 2.0 ** -22 * (rows + 2) * np.abs(ref) + 1e-30
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()


@pytest.mark.parametrize("kind", ["bf16", "e2m1"])
@pytest.mark.parametrize("sizes", [[5, 0], [0, 5, 0], [0, 4, 0, 0]])
def test_a_path_through_no_tree_adds_nothing(torch, sizes, kind):
    """Sequences without rows whose path has entries all the same: none is a row, the last sequence's would lie behind q and lse."""
    from paper_2510_26577_amd import cache4, evict
    rng = np.random.default_rng(len(sizes))
    Hq, Hkv, D, L, n = 8, 2, 128, 70, 3
    B, rows = len(sizes), sum(sizes)
    lay = cc.Layout(rng, [L] * B, Hkv, D, 16)
    if kind == "e2m1":
        four = cc.FourBit(rng, lay, [L] * B)
        cache, K = four.cache, [four.values(b, np.arange(L))[0] for b in range(B)]
    else:
        x = orc.to_bf16(rng.standard_normal((lay.rows, D)))
        cache, K = lay.cache(kind=cache4.ROWS_BF16, k=cc.dev(x)), [orc.bf16(x[lay.at(b, np.arange(L))]) for b in range(B)]
    q = orc.to_bf16(rng.standard_normal((rows, Hq, D)))
    lse = (rng.random((rows, Hq)) * 3 + 3).astype(np.float32)
    w0 = rng.random((B, Hkv, L)).astype(np.float32)
    w, pos = cc.dev(w0), torch.full((B, Hkv, L), -3, dtype=torch.int32, device="cuda")
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    path = np.tile(np.arange(n, dtype=np.int32), (B, 1))
    evict.key_weights(q=cc.dev(q), lse=cc.dev(lse), cache=cache, cu_T=cc.dev(cu), L=cc.dev([L] * B, np.int32), weight=w, max_rows=n, max_L=L, scale=0.1,
                      path=cc.dev(path), path_len=cc.dev([n] * B, np.int32), pos=pos, first_pos=cc.dev(np.arange(B) * 100, np.int32))
    torch.cuda.synchronize()
    got = w.cpu().numpy()
    for b in range(B):
        at = cu[b] + np.arange(n)
        l = lse[at].astype(np.float64) if sizes[b] else np.full((n, Hq), -np.inf)
        ref, off = orc.key_weights(w0[b], orc.bf16(q[at]) if sizes[b] else np.zeros((n, Hq, D)), l, K[b], n, 0.1)
        _close(got[b], ref, off, n * Hq // Hkv)
        assert (pos[b, :, L - n:].cpu().numpy() == b * 100 + np.arange(n)).all() and (pos[b, :, :L - n] == -3).all()


@pytest.mark.parametrize("heads,n,page", [((4, 4, 64), 3, 0), ((8, 2, 128), 5, 16), ((24, 8, 128), 32, 16), ((8, 8, 128), 33, 0), ((32, 8, 64), 1, 5)])
@pytest.mark.parametrize("rows", ["bf16", "e4m3"])
def test_keys_that_are_not_finite_weigh_what_the_rows_give_them(torch, heads, n, page, rows):
    """Infinities and NaN among a sequence's own keys, old ones and new ones, beside rows that add nothing: padding of a block of 32,
    lse = -inf, path entries that are no rows.  A row that counts gives exp(+-inf) or NaN, the others nothing."""
    from paper_2510_26577_amd import cache4, evict
    rng = np.random.default_rng(n + page)
    Hq, Hkv, D = heads
    G, L, T = Hq // Hkv, 150, n + 4
    lay = cc.Layout(rng, [L], Hkv, D, page)
    at = lay.at(0, np.arange(L))
    keys = [3, 40, 64, 149 - n, 149]  # blocks that all rows see, and those of the newest rows
    if rows == "e4m3":
        x = torch.from_numpy(rng.standard_normal((lay.rows, D)).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy().copy()
        for i, t in enumerate(keys):
            x[at[t, i % Hkv], 5 * i] = (0x7F, 0xFF)[i % 2]  # (the format has no infinities)
        K = torch.from_numpy(x).view(torch.float8_e4m3fn).double().numpy()[at]
        cache = lay.cache(kind=cache4.ROWS_E4M3, k=cc.dev(x))
    else:
        x = orc.to_bf16(rng.standard_normal((lay.rows, D)))
        for i, t in enumerate(keys):
            x[at[t, i % Hkv], 5 * i] = (0x7F80, 0xFF80, 0x7FC0)[i % 3]
        K = orc.bf16(x[at])
        cache = lay.cache(kind=cache4.ROWS_BF16, k=cc.dev(x))
    q = orc.to_bf16(rng.standard_normal((T, Hq, D)))
    lse = (rng.random((T, Hq)) * 3 + 3).astype(np.float32)
    path = np.sort(rng.choice(T, n, replace=False)).astype(np.int32)
    for case in ("some", "none"):
        off_rows = rng.random((T, Hq)) < (0.2 if case == "some" else 2.0)
        l = np.where(off_rows, -np.inf, lse).astype(np.float32)
        w0 = rng.random((1, Hkv, L)).astype(np.float32)
        w, p = cc.dev(w0), path.copy()
        if n > 2:
            p[1] = T  # no row
        evict.key_weights(q=cc.dev(q), lse=cc.dev(l), cache=cache, cu_T=cc.dev([0, T], np.int32), L=cc.dev([L], np.int32), weight=w, max_rows=n, max_L=L,
                          scale=0.1, path=cc.dev(p[None]), path_len=cc.dev([n], np.int32))
        got = w.cpu().numpy()[0].astype(np.float64)
        ls = np.where((p < T)[:, None], l[np.minimum(p, T - 1)].astype(np.float64), -np.inf)
        with np.errstate(invalid="ignore", over="ignore"):
            ref, off = orc.key_weights(w0[0], orc.bf16(q[np.minimum(p, T - 1)]), ls, K, n, 0.1)
        fine = np.isfinite(ref)
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]) and np.isfinite(got[fine]).all()
        assert case == "some" or fine.all()
        off = np.where(np.isfinite(off), off, 0.0)  # (a weight of exp(-inf), exactly 0: its bound is 0 * inf)
        _close(got[fine], ref[fine], off[fine], n * G)
