"""GPU tests of tva_rotate and tva_cache_append against the definition in 64 bits (oracle/layer_oracle.py)."""
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


H = {"4/4/64": (4, 4, 64), "24/8/128": (24, 8, 128), "32/8/128": (32, 8, 128), "32/8/64": (32, 8, 64), "16/1/128": (16, 1, 128), "5/3/128": (5, 3, 128),
     "71/9/64": (71, 9, 64)}


def bound(want, size):
    """The result is rounded to bf16 once (half a step, 2^-8 of it, or of the smallest normal number).  Before that: sine and cosine are off
    by 4 steps of 2^-24 and by what the fp32 turns leave of the angle, 2 pi 2^-25; a norm sums 128 squares and takes a root and two
    quotients; two products and a sum: together below 2^-18 of the terms."""
    return 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size + 2.0 ** -133


def check(got, want, size):
    off = np.abs(got - want)
    assert (off <= bound(want, size)).all(), ((off - bound(want, size)).max(), np.unravel_index((off / bound(want, size)).argmax(), off.shape))


def wide(torch, rng, n, heads, spare=0):
    """A projection's output: q, k and v heads side by side, `spare` more columns (of 8 elements) and a row behind the last."""
    Hq, Hkv, D = heads
    width = (Hq + 2 * Hkv) * D + 8 * spare
    x = to_bf16(rng.standard_normal((n + 1, width)) * 2.0)
    d = cc.dev(x)
    cut = lambda a, h: (x[:, a * D:(a + h) * D].reshape(n + 1, h, D)[:n], d[:, a * D:(a + h) * D].unflatten(1, (h, D))[:n])  # noqa: E731
    return cut(0, Hq), cut(Hq, Hkv), cut(Hq + Hkv, Hkv), d


def sequences(rng, sizes, lengths, tree):
    cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    words = 1 + (max(sizes) > 64)
    if not tree:
        return cu, np.concatenate([L + np.arange(T) for T, L in zip(sizes, lengths)] + [[]]).astype(np.int64), None
    sets = [cc.ancestor_sets(p) for p in cc.trees(rng, sizes)]
    mask = np.concatenate([cc.mask_words(s, words) for s in sets])
    return cu, np.concatenate([L + s.sum(1) - 1 for L, s in zip(lengths, sets)]).astype(np.int64), mask


def _rotate(torch, rng, heads, sizes, lengths, dims, interleaved=False, norm=False, tree=False, scaling=0, spare=0, in_place=False, pos=None, which="qk", magnitude=None):
    from paper_2510_26577_amd import rotary
    Hq, Hkv, D = heads
    cu, where, mask = sequences(rng, sizes, lengths, tree)
    n = int(cu[-1])
    (q, dq), (k, dk), _, x = wide(torch, rng, n, heads, spare)
    before = x.clone()
    freq, m = rotary.frequencies(max(dims, 4), scaling=scaling, factor=4.0, original=4096.0)
    freq, m = freq[:dims // 2], m if magnitude is None else magnitude
    norms = [to_bf16(1 + 0.3 * rng.standard_normal(D)) for _ in range(2)] if norm else [None, None]
    outs = [dq, dk] if in_place else [torch.full((n + 1, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv)]
    kw = dict(freq=cc.dev(freq) if dims else None, dims=dims, interleaved=interleaved, magnitude=m, eps=1e-5, cu_T=cc.dev(cu), L=cc.dev(np.array(lengths, np.int32)),
              anc_mask=None if mask is None else cc.dev(mask))
    if pos is not None:
        where = np.asarray(pos)
        kw["pos"] = cc.dev(where, np.int32)
    if "q" in which:
        kw.update(q=dq, q_out=outs[0], q_norm=None if norms[0] is None else cc.dev(norms[0]))
    if "k" in which:
        kw.update(k=dk, k_out=outs[1], k_norm=None if norms[1] is None else cc.dev(norms[1]))
    rotary.rotate(**kw)
    torch.cuda.synchronize()
    for name, a, w, o in (("q", q, norms[0], outs[0]), ("k", k, norms[1], outs[1])):
        if name not in which:
            assert in_place or (o == 7).all()
            continue
        want, size = orc.heads(bf16(a), where, freq, dims, interleaved, m, None if w is None else bf16(w), 1e-5)
        check(bf16(cc.bits(o))[:n], want, size)
        if not in_place:
            assert (o[n] == 7).all()
    if not in_place:
        assert torch.equal(x.view(torch.int16), before.view(torch.int16))
    else:  # the rest of the projection stays
        cols = (Hq + Hkv) * D
        assert torch.equal(x[:, cols:].view(torch.int16), before[:, cols:].view(torch.int16)) and torch.equal(x[n].view(torch.int16), before[n].view(torch.int16))
    return kw


@pytest.mark.parametrize("heads", list(H))
@pytest.mark.parametrize("norm,interleaved", [(False, False), (True, False), (False, True), (True, True)])
def test_heads_over_shapes(torch, heads, norm, interleaved):
    _rotate(torch, np.random.default_rng(1), H[heads], [5, 1, 17], [100, 0, 3000], H[heads][2], interleaved, norm)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dims", [0, 16, 32, 48, 64, 80, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_of_a_head(torch, D, dims, interleaved):
    if dims <= D:
        _rotate(torch, np.random.default_rng(dims), (8, 2, D), [9], [777], dims, interleaved, dims % 32 == 0)


@pytest.mark.parametrize("scaling", range(5))
@pytest.mark.parametrize("L", [0, 1, 131071, 1 << 20, (1 << 30) - 40])
def test_positions_near_and_far(torch, scaling, L):
    _rotate(torch, np.random.default_rng(L % 97), (4, 2, 128), [30, 2], [L, L // 2], 128, scaling == 3, scaling=scaling)


@pytest.mark.parametrize("sizes", [[1], [2], [64], [128], [60, 1, 100], [3] * 70, [1] * 200])
def test_trees_positions_are_depths(torch, sizes):
    rng = np.random.default_rng(len(sizes))
    _rotate(torch, rng, (8, 2, 64), sizes, rng.integers(0, 5000, len(sizes)).tolist(), 64, tree=True, norm=True)


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 129, 4097])
def test_rows_find_their_sequence(torch, B):
    rng = np.random.default_rng(B)
    sizes = rng.integers(0, 3, B)
    sizes[rng.integers(0, B)] += 2
    _rotate(torch, rng, (2, 1, 64), sizes.tolist(), rng.integers(0, 100000, B).tolist(), 16)


def test_positions_that_are_given(torch):
    rng = np.random.default_rng(3)
    pos = [-5, 0, 7, 1 << 30, -(1 << 31), (1 << 31) - 1, 3, 3]
    _rotate(torch, rng, (4, 4, 128), [8], [9], 128, pos=pos)
    from paper_2510_26577_amd import rotary  # without sequences
    x = to_bf16(rng.standard_normal((8, 4, 128)))
    freq, _ = rotary.frequencies(128)
    out, none = rotary.rotate(q=cc.dev(x), pos=cc.dev(pos, np.int32), freq=cc.dev(freq), dims=128)
    want, size = orc.heads(bf16(x), pos, freq, 128)
    assert none is None
    check(bf16(cc.bits(out)), want, size)


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_one_of_the_two_in_place_and_strides(torch, which, in_place, interleaved):
    _rotate(torch, np.random.default_rng(4), (6, 2, 128), [33, 4], [10, 20], 96, interleaved, True, spare=3, in_place=in_place, which=which)


@pytest.mark.parametrize("heads", ["32/8/128", "71/9/64", "5/3/128"])
def test_in_place_over_more_rows_than_a_wave_has_on_the_way(torch, heads):
    _rotate(torch, np.random.default_rng(5), H[heads], [70, 3], [0, 9], H[heads][2], False, True, in_place=True)


def test_rows_behind_the_last_sequence_are_left(torch):
    from paper_2510_26577_amd import rotary
    x = torch.randn(9, 4, 64, device="cuda").bfloat16()
    out = torch.full_like(x, 7.0)
    freq = cc.dev(rotary.frequencies(64)[0])
    for cu, used in (([0, 2, 5], 5), ([0, 0, 0], 0), ([0, 9, 9], 9)):
        out.fill_(7.0)
        rotary.rotate(q=x, q_out=out, cu_T=cc.dev(cu, np.int32), L=cc.dev([3, 4], np.int32), freq=freq, dims=64)
        assert (out[used:] == 7).all() and (out[:used] != 7).any() == (used > 0)


def test_values_that_are_not_finite_stay_in_their_pairs(torch):
    from paper_2510_26577_amd import rotary
    x = torch.randn(2, 2, 128, device="cuda").bfloat16()
    x[0, 0, 3], x[0, 1, 100] = float("inf"), float("nan")
    freq = cc.dev(rotary.frequencies(64)[0])
    out, _ = rotary.rotate(q=x, pos=cc.dev([5, 6], np.int32), freq=freq, dims=64)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[0, 0, 3] = want[0, 0, 35] = want[0, 1, 100] = True
    assert torch.equal(bad, want)


# ---- append ----
def _stores(torch, kind, lay):
    """Empty caches: (tensors for make_cache, what they hold)."""
    D, n = lay.D, lay.rows
    if kind == "bf16":
        return dict(kind=0, **{x: torch.full((n, D), 7.0, dtype=torch.bfloat16, device="cuda") for x in "kv"})
    if kind == "e4m3":
        return dict(kind=1, k_scale=0.02, v_scale=0.013, **{x: torch.full((n, D), 0x35, dtype=torch.uint8, device="cuda") for x in "kv"})
    return dict(kind=2, **{x: torch.full((n, D // 2), 0x35, dtype=torch.uint8, device="cuda") for x in "kv"},
                k_row_scale=torch.full((n, D // 32), 9, dtype=torch.uint8, device="cuda"), v_row_scale=torch.full((n,), 7.0, dtype=torch.bfloat16, device="cuda"))


def _append(torch, rng, heads, sizes, lengths, rows, page=0, head_major=False, tree=False, norm=False, interleaved=False, dims=None, with_q=True, k_out=False, room=None,
            stream=None, magnitude=1.0):
    """The cache against the rows that tva_rotate gives (checked above), rounded as defined."""
    from paper_2510_26577_amd import rotary
    Hq, Hkv, D = heads
    dims = D if dims is None else dims
    cu, where, mask = sequences(rng, sizes, lengths, tree)
    n, B = int(cu[-1]), len(sizes)
    (q, dq), (k, dk), (v, dv), x = wide(torch, rng, n, heads, 2)
    room = [L + T for L, T in zip(lengths, sizes)] if room is None else room
    lay = cc.Layout(rng, room, Hkv, D, page, head_major)
    held = _stores(torch, rows, lay)
    before = {name: t.clone() for name, t in held.items() if hasattr(t, "clone")}
    freq, _ = rotary.frequencies(D)
    norms = [cc.dev(to_bf16(1 + 0.3 * rng.standard_normal(D))) if norm else None for _ in range(2)]
    both = dict(freq=cc.dev(freq[:max(1, dims // 2)]), dims=dims, interleaved=interleaved, magnitude=magnitude, eps=1e-5, cu_T=cc.dev(cu),
                L=cc.dev(np.array(lengths, np.int32)), anc_mask=None if mask is None else cc.dev(mask))
    turned_q, turned = rotary.rotate(q=dq, k=dk, q_norm=norms[0], k_norm=norms[1], **both)
    L_out, flag = torch.full((B,), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    more = dict(k_out=torch.zeros_like(turned)) if k_out else {}
    if with_q:
        more.update(q=dq, q_norm=norms[0])
    torch.cuda.synchronize()
    out = rotary.append(k=dk, v=dv, k_norm=norms[1], cache=lay.cache(**held), L_out=L_out, err_flag=flag, stream=stream, **more, **both)
    torch.cuda.synchronize()
    same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))  # noqa: E731
    assert same(out, turned_q) if with_q else out is None
    assert not k_out or same(more["k_out"], turned)
    assert L_out.tolist() == [L + T for L, T in zip(lengths, sizes)]
    left = {name: t.cpu().clone() for name, t in before.items()}
    missed = set()
    kt, vt = cc.bits(turned), v
    for b in range(B):
        there = [i for i in range(sizes[b]) if lengths[b] + i < (room[b] if not page else lay.table.shape[1] * page)]
        if len(there) < sizes[b]:
            missed.add(1 + b)
        if not there:
            continue
        at = lay.at(b, lengths[b] + np.array(there))
        r = cu[b] + np.array(there)
        if rows == "bf16":
            new = dict(k=torch.from_numpy(kt[r].view(np.int16)).view(torch.bfloat16), v=torch.from_numpy(vt[r].view(np.int16).copy()).view(torch.bfloat16))
        elif rows == "e4m3":
            new = dict(k=torch.from_numpy(orc.eight_bit(bf16(kt[r]), 0.02)), v=torch.from_numpy(orc.eight_bit(bf16(vt[r]), 0.013)))
        else:
            a, s, c, d = cache_oracle.encode_rows(kt[r], vt[r])
            new = dict(k=torch.from_numpy(a), k_row_scale=torch.from_numpy(s), v=torch.from_numpy(c), v_row_scale=torch.from_numpy(d.view(np.int16)).view(torch.bfloat16))
        for name, t in new.items():
            left[name][torch.from_numpy(at)] = t
    for name, t in left.items():
        here = same(held[name].cpu(), t)
        assert here, name
    assert (int(flag) in missed) if missed else int(flag) == 0


@pytest.mark.parametrize("rows", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("heads", ["4/4/64", "32/8/128", "5/3/128", "16/1/128", "71/9/64"])
@pytest.mark.parametrize("page,head_major", [(0, False), (0, True), (16, False), (5, True)])
def test_append_over_heads_and_layouts(torch, rows, heads, page, head_major):
    _append(torch, np.random.default_rng(1), H[heads], [13, 1, 6], [50, 3, 0], rows, page, head_major)


@pytest.mark.parametrize("rows", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("kw", [dict(tree=True), dict(norm=True, k_out=True), dict(interleaved=True, dims=32, with_q=False), dict(dims=0, norm=True), dict(magnitude=1.3)])
def test_append_of_trees_norms_and_parts(torch, rows, kw):
    _append(torch, np.random.default_rng(2), (8, 2, 64 if kw.get("tree") else 128), [9, 0, 30], [7, 4, 100], rows, 16, **kw)


@pytest.mark.parametrize("rows", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("page", [0, 8])
def test_positions_without_a_place_are_left_out(torch, rows, page):
    room = [24, 24, 24] if page else [5, 13, 24]  # (a page table's rows are equally long, and all their entries are pages)
    _append(torch, np.random.default_rng(3), (4, 2, 64), [10, 3, 4], [16, 10, 20], rows, page, room=[24, 24, 24])
    _append(torch, np.random.default_rng(4), (4, 2, 64), [10, 3, 4], [2, 10, 30], rows, page, room=room)
    _append(torch, np.random.default_rng(5), (4, 2, 64), [10, 3, 4], [20, 22, 1 << 30], rows, page, room=room)


def test_lengths_are_written_without_rows(torch):
    from paper_2510_26577_amd import rotary
    k = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")[:0]
    lay = cc.Layout(np.random.default_rng(0), [4, 4], 2, 64)
    L_out = torch.zeros(2, dtype=torch.int32, device="cuda")
    rotary.append(k=k, v=k, cache=lay.cache(**_stores(torch, "bf16", lay)), cu_T=cc.dev([0, 0, 0], np.int32), L=cc.dev([3, 1], np.int32), dims=0, L_out=L_out)
    assert L_out.tolist() == [3, 1]


def test_every_eight_bit_code_and_its_borders(torch):
    """All bf16 numbers, finite or not, through the 8-bit rounding with two scales."""
    from paper_2510_26577_amd import rotary
    x = np.arange(65536, dtype=np.uint16).reshape(-1, 2, 128)
    n = len(x)
    d, lay = cc.dev(x), cc.Layout(np.random.default_rng(0), [n], 2, 128)
    for scale in (1.0, 0.37):
        held = dict(_stores(torch, "e4m3", lay), k_scale=scale, v_scale=1.0)
        rotary.append(k=d, v=d, cache=lay.cache(**held), cu_T=cc.dev([0, n], np.int32), L=cc.dev([0], np.int32), dims=0)
        at = lay.at(0, np.arange(n))
        codes = {c: orc.eight_bit(bf16(x), c) for c in {scale, 1.0}}
        assert np.array_equal(held["k"].cpu().numpy()[at], codes[scale])
        assert np.array_equal(held["v"].cpu().numpy()[at], codes[1.0])


@pytest.mark.parametrize("rows", ["bf16", "e2m1"])
def test_append_on_another_stream(torch, rows):
    s = torch.cuda.Stream()
    _append(torch, np.random.default_rng(6), (32, 8, 128), [700], [5], rows, 16, stream=s)
