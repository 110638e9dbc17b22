"""What the Python calls of rotary.py and chunk.py refuse, and the library's own checks of include/tva_layer.h: all before anything is queued (CPU)."""
import ctypes

import pytest
import torch

from paper_2510_26577_amd import binding, cache4, chunk, rotary
from tests.test_abi import declared_symbols

BF, F, I = torch.bfloat16, torch.float32, torch.int32
B, T, HQ, HKV, D = 2, 3, 4, 2, 64
N = B * T


def _t(*shape, dtype=F, device="cpu"):
    return torch.zeros(shape, dtype=dtype, device=device)


def _cache(**kw):
    return cache4.make_cache(**dict(dict(kind=0, k=_t(64, D, dtype=BF), v=_t(64, D, dtype=BF), cu_L=_t(B + 1, dtype=I)), **kw))


def _rotate(**kw):
    return dict(dict(q=_t(N, HQ, D, dtype=BF), k=_t(N, HKV, D, dtype=BF), q_out=_t(N, HQ, D, dtype=BF), k_out=_t(N, HKV, D, dtype=BF),
                     freq=_t(D // 2, dtype=torch.float64), dims=D, cu_T=_t(B + 1, dtype=I), L=_t(B, dtype=I), q_norm=_t(D, dtype=BF), k_norm=_t(D, dtype=BF),
                     anc_mask=_t(N, 1, dtype=torch.int64)), **kw)


def _append(**kw):
    return dict(dict(_rotate(), v=_t(N, HKV, D, dtype=BF), cache=_cache(), L_out=_t(B, dtype=I), err_flag=_t(1, dtype=I)), **kw)


def _attn(**kw):
    return dict(dict(q=_t(N, HQ, D, dtype=BF), cache=_cache(), cu_T=_t(B + 1, dtype=I), L=_t(B, dtype=I), Hkv=HKV, max_T=T, max_L=20, scale=1.0,
                     anc_mask=_t(N, 1, dtype=torch.int64), out=_t(N, HQ, D, dtype=BF), lse=_t(N, HQ), workspace=_t(4)), **kw)


MAKE = {"rotate": (rotary.make_rotate_args, _rotate), "append": (rotary.make_append_args, _append), "attn": (chunk.make_args, _attn)}
FN = {"rotate": "tva_rotate", "append": "tva_cache_append", "attn": "tva_chunk_attn"}


def make(which, **kw):
    f, args = MAKE[which]
    return f(**args(**kw))


def test_layer_exports_match_header():
    lib = binding.load_library()
    syms = declared_symbols("tva_layer.h")
    assert set(syms) == set(binding.LAYER_EXPORTS)
    for s in syms:
        assert getattr(lib, s) is not None
    assert lib.tva_sizeof_rotate_args() == ctypes.sizeof(rotary.RotateArgs)
    assert lib.tva_sizeof_append_args() == ctypes.sizeof(rotary.AppendArgs)
    assert lib.tva_sizeof_chunk_args() == ctypes.sizeof(chunk.ChunkArgs)


@pytest.mark.parametrize("which", list(MAKE))
def test_what_is_right_is_taken(which):
    make(which)


HALF = _t(2 * N, HQ, D, dtype=BF)[::2]  # rows further apart: a stride


@pytest.mark.parametrize("which,kw", [
    ("rotate", dict(q=_t(N, HQ, D))), ("rotate", dict(q=_t(N, HQ * D, dtype=BF))), ("rotate", dict(q=_t(N, D, HQ, dtype=BF).transpose(1, 2))),
    ("rotate", dict(q_out=None)), ("rotate", dict(k_out=None)), ("rotate", dict(q=None)), ("rotate", dict(q_out=_t(N - 1, HQ, D, dtype=BF))),
    ("rotate", dict(k_out=_t(N, HQ, D, dtype=BF))), ("rotate", dict(k=_t(N - 1, HKV, D, dtype=BF))), ("rotate", dict(freq=_t(D // 2))),
    ("rotate", dict(freq=None)), ("rotate", dict(freq=_t(D // 2 - 1, dtype=torch.float64))), ("rotate", dict(q_norm=_t(D))), ("rotate", dict(k_norm=_t(D // 2, dtype=BF))),
    ("rotate", dict(cu_T=None)), ("rotate", dict(L=None)), ("rotate", dict(L=_t(B - 1, dtype=I))), ("rotate", dict(L=_t(B, dtype=torch.int64))),
    ("rotate", dict(pos=_t(N - 1, dtype=I))), ("rotate", dict(pos=_t(N))), ("rotate", dict(anc_mask=_t(N - 1, 1, dtype=torch.int64))),
    ("rotate", dict(anc_mask=_t(N, 1, dtype=I))), ("rotate", dict(q=None, k=None, q_out=None, k_out=None)),
    ("rotate", dict(q=_t(N, HQ * D + 4, dtype=BF)[:, :HQ * D].unflatten(1, (HQ, D)))), ("rotate", dict(q=_t(1, HQ, D, dtype=BF).expand(N, HQ, D))),
    ("rotate", dict(freq=_t(D // 2, dtype=torch.float64, device="meta"))),
    ("append", dict(v=_t(N, HQ, D, dtype=BF))), ("append", dict(v=_t(N, HKV, D))), ("append", dict(L_out=_t(B - 1, dtype=I))), ("append", dict(cu_T=None)), ("append", dict(L=None)),
    ("append", dict(cache=_cache(cu_L=_t(B, dtype=I)))), ("append", dict(err_flag=_t(1))), ("append", dict(cache=_cache(cu_L=None, page_table=_t(1, 4, dtype=I), page_size=16))),
    ("attn", dict(q=_t(N, HQ, D))), ("attn", dict(out=_t(N, HQ, D))), ("attn", dict(out=_t(N - 1, HQ, D, dtype=BF))), ("attn", dict(lse=_t(N, HQ + 1))), ("attn", dict(lse=_t(N * HQ))),
    ("attn", dict(out=_t(N, D, HQ, dtype=BF).transpose(1, 2))), ("attn", dict(anc_mask=_t(N - 1, 1, dtype=torch.int64))), ("attn", dict(L=_t(1, dtype=I))),
    ("attn", dict(cu_T=_t(B + 1))), ("attn", dict(workspace=_t(4, 4).T[:, 1:])), ("attn", dict(cache=_cache(cu_L=_t(B, dtype=I)))), ("attn", dict(lse=_t(N, HQ, dtype=BF))),
])
def test_tensors_the_kernels_would_take_for_others_are_refused(which, kw):
    with pytest.raises(ValueError):
        make(which, **kw)


def test_rows_that_lie_further_apart_are_told_by_their_stride():
    a = make("rotate", q=HALF, q_out=_t(N, HQ, D, dtype=BF))
    assert a.q_stride == 2 * HQ * D and a.q_out_stride == HQ * D
    x = _t(N, (HQ + 2 * HKV) * D + 8, dtype=BF)
    a = make("append", k=x[:, HQ * D:(HQ + HKV) * D].unflatten(1, (HKV, D)), v=x[:, (HQ + HKV) * D:(HQ + 2 * HKV) * D].unflatten(1, (HKV, D)))
    assert a.r.k_stride == a.v_stride == (HQ + 2 * HKV) * D + 8
    assert make("attn", q=HALF).q_stride == 2 * HQ * D


@pytest.mark.parametrize("which", list(MAKE))
def test_host_tensors_are_refused(which):
    f = {"rotate": rotary.rotate, "append": rotary.append, "attn": lambda **kw: chunk.attn(kw.pop("q"), kw.pop("cache"), kw.pop("cu_T"), kw.pop("L"), **kw)}[which]
    with pytest.raises(ValueError, match="GPU"):
        f(**MAKE[which][1]())


def status(which, **fields):
    """The library's answer to a block with some fields changed (nested as r.x and cache.x); nothing may be queued."""
    a = make(which)
    for name, v in fields.items():
        at, path = a, name.split("__")
        for part in path[:-1]:
            at = getattr(at, part)
        setattr(at, path[-1], v)
    return getattr(binding.load_library(), FN[which])(ctypes.byref(a), None)


@pytest.mark.parametrize("which,fields,want", [
    ("rotate", dict(D=96), -2), ("rotate", dict(dims=24), -2), ("rotate", dict(dims=80), -1), ("rotate", dict(dims=-16), -1), ("rotate", dict(eps=-1.0), -1),
    ("rotate", dict(eps=float("nan")), -1), ("rotate", dict(magnitude=float("inf")), -1), ("rotate", dict(B=-1), -1), ("rotate", dict(sum_T=-1), -1), ("rotate", dict(Hq=0), -1),
    ("rotate", dict(q_out=None), -1), ("rotate", dict(k_out=None), -1), ("rotate", dict(q=None, k=None), -1), ("rotate", dict(freq=None), -1), ("rotate", dict(L=None), -1),
    ("rotate", dict(cu_T=None), -1), ("rotate", dict(mask_words=3), -2), ("rotate", dict(q_stride=HQ * D - 8), -1), ("rotate", dict(k_out_stride=HKV * D + 4), -1),
    ("rotate", dict(q=24), -1), ("rotate", dict(k_norm=8), -1), ("rotate", dict(q_out_stride=-8), -1), ("rotate", dict(q=64, q_out=64, q_out_stride=HQ * D + 8), -1),
    ("append", dict(r__k=None, r__k_out=None), -1), ("append", dict(v=None), -1), ("append", dict(v=8), -1), ("append", dict(v_stride=4), -1), ("append", dict(r__L=None), -1),
    ("append", dict(cache__kind=3), -1), ("append", dict(cache__kind=2), -1), ("append", dict(cache__cu_L=None), -1), ("append", dict(cache__stride_tok=4), -1), ("append", dict(r__dims=8), -2),
    ("attn", dict(B=0), -1), ("attn", dict(Hkv=3), -1), ("attn", dict(D=32), -2), ("attn", dict(scale=0.0), -1), ("attn", dict(window=-1), -1), ("attn", dict(n_first=-1), -1),
    ("attn", dict(num_splits=-1), -1), ("attn", dict(plan_rows=64), -1), ("attn", dict(max_T=129), -2), ("attn", dict(mask_words=0), -2), ("attn", dict(cache__kind=2), -2),
    ("attn", dict(cache__kind=9), -1), ("attn", dict(q_stride=8), -1), ("attn", dict(q_stride=HQ * D + 4), -1), ("attn", dict(q=None), -1), ("attn", dict(out=None), -1),
    ("attn", dict(L=None), -1), ("attn", dict(q=8), -1), ("attn", dict(max_L=1 << 30), -2), ("attn", dict(anc_mask=None, max_T=1 << 29), -2), ("attn", dict(workspace=8, workspace_bytes=1 << 30, num_splits=2, max_L=4000), -1),
    ("attn", dict(workspace_bytes=4, num_splits=2, workspace=64, max_L=4000), -3), ("attn", dict(cache__page_table=64), -1), ("attn", dict(cache__v=None), -1),
])
def test_blocks_the_library_refuses(which, fields, want):
    assert status(which, **fields) == want


def test_lengths_that_come_back_where_they_were_read_are_refused():
    a = make("append")
    a.L_out = a.r.L
    assert binding.load_library().tva_cache_append(ctypes.byref(a), None) == -1


@pytest.mark.parametrize("which,fields", [("rotate", dict(sum_T=0)), ("rotate", dict(B=0)), ("append", dict(r__sum_T=0, L_out=None)), ("append", dict(r__B=0)),
                                          ("attn", dict(sum_T=0)), ("attn", dict(max_T=0))])
def test_nothing_to_do_is_no_error(which, fields):
    assert status(which, **fields) == 0


def shape(**kw):
    a = chunk.ChunkArgs()
    a.B, a.Hq, a.Hkv, a.D, a.sum_T, a.max_T, a.max_L = 1, 32, 8, 128, 1, 1, 4096
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_plan_and_workspace():
    assert chunk.plan_rows(shape()) == 32 and chunk.plan_rows(shape(plan_rows=128)) == 128
    assert chunk.plan_rows(shape(sum_T=4096, max_T=4096)) >= 128
    assert chunk.plan_splits(shape()) > 1 and chunk.plan_splits(shape(num_splits=1)) == 1
    assert chunk.workspace_bytes(shape(num_splits=1)) == 0
    n = chunk.plan_splits(shape(num_splits=4))
    assert n <= 4 and chunk.workspace_bytes(shape(num_splits=4)) % (n * 8 * 32 * 129 * 4) == 0
    assert chunk.plan_splits(shape(max_L=0)) == 1          # one tile
    assert chunk.plan_splits(shape(max_L=100000, window=64, n_first=4)) <= 4  # as many as the window has tiles
    assert chunk.plan_splits(shape(B=64, sum_T=64 * 2048, max_T=2048)) == 1
    for bad in (dict(D=80), dict(Hkv=5), dict(B=0), dict(window=-1)):
        for f in (chunk.plan_rows, chunk.plan_splits, chunk.workspace_bytes):
            with pytest.raises(binding.TvaError):
                f(shape(**bad))
