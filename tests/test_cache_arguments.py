"""What the Python calls of cache4.py and evict.py refuse: tensors whose type, length or place the kernels would take for another (CPU)."""
import numpy as np
import pytest
import torch

from paper_2510_26577_amd import cache4, evict

BF, F, I = torch.bfloat16, torch.float32, torch.int32
B, T, HQ, HKV, D, LD = 2, 3, 4, 2, 64, 24


def _t(*shape, dtype=F, device="cpu"):
    return torch.zeros(shape, dtype=dtype, device=device)


def _cache(**kw):
    return dict(dict(k=_t(64, 32, dtype=torch.uint8), v=_t(64, 32, dtype=torch.uint8), k_row_scale=_t(64, 2, dtype=torch.uint8),
                     v_row_scale=_t(64, dtype=BF), cu_L=_t(B + 1, dtype=I)), **kw)


def _paged(**kw):
    return _cache(**dict(dict(cu_L=None, page_table=_t(B, 4, dtype=I), page_size=8), **kw))


def _rows(**kw):
    return dict(dict(k_rows=_t(B * T, HKV, D, dtype=BF), v_rows=_t(B * T, HKV, D, dtype=BF), cu_T=_t(B + 1, dtype=I), L=_t(B, dtype=I), max_rows=T,
                     path=_t(B, T, dtype=I), path_len=_t(B, dtype=I), L_out=_t(B, dtype=I)), **kw)


def _attn(**kw):
    return dict(dict(q=_t(B * T, HQ, D, dtype=BF), k_tree=_t(B * T, HKV, D, dtype=BF), v_tree=_t(B * T, HKV, D, dtype=BF), cu_T=_t(B + 1, dtype=I),
                     L=_t(B, dtype=I), max_T=T, max_L=LD, scale=1.0, anc_mask=_t(B * T, 1, dtype=torch.int64), out=_t(B * T, HQ, D, dtype=BF),
                     lse=_t(B * T, HQ), workspace=_t(4)), **kw)


def _weigh(**kw):
    return dict(dict(q=_t(B * T, HQ, D, dtype=BF), lse=_t(B * T, HQ), cu_T=_t(B + 1, dtype=I), L=_t(B, dtype=I), weight=_t(B, HKV, LD), max_rows=T,
                     max_L=LD, scale=1.0, path=_t(B, T, dtype=I), path_len=_t(B, dtype=I), pos=_t(B, HKV, LD, dtype=I), first_pos=_t(B, dtype=I)), **kw)


def _select(**kw):
    return dict(dict(weight=_t(B, HKV, LD), L=_t(B, dtype=I), keep=_t(B, dtype=I), max_L=LD, src=_t(B, HKV, LD, dtype=I), L_out=_t(B, dtype=I),
                     newest=_t(B, dtype=I), pos=_t(B, HKV, LD, dtype=I)), **kw)


def _move(**kw):
    return dict(dict(src=_t(B, HKV, LD, dtype=I), n=_t(B, dtype=I), Hkv=HKV, D=D, max_keep=LD, weight=_t(B, HKV, LD), pos=_t(B, HKV, LD, dtype=I)), **kw)


def _make(which, cache=None, **kw):
    if which == "cache":
        return cache4.make_cache(**_cache(**kw))
    if which == "select":
        return evict.make_select_args(**_select(**kw))
    c = cache4.make_cache(**(_cache() if cache is None else cache))
    make, args = {"rows": (cache4.make_rows_args, _rows), "attn": (cache4.make_attn_args, _attn), "weigh": (evict.make_key_weight_args, _weigh),
                  "move": (evict.make_move_args, _move)}[which]
    return make(cache=c, **args(**kw))


def test_arguments_that_fit_are_taken():
    for which in ("cache", "rows", "attn", "weigh", "select", "move"):
        _make(which)
    for which in ("rows", "attn", "weigh", "move"):
        _make(which, _paged())
    _make("attn", anc_mask=None, parent=_t(B * T, dtype=I), out=_t(B * T + 2, HQ, D, dtype=BF), lse=None)
    _make("attn", anc_mask=_t(B * T, 1, dtype=torch.uint64))
    _make("rows", path=None, path_len=None, L_out=None)
    for kind, dtypes in ((cache4.ROWS_BF16, (BF,)), (cache4.ROWS_E4M3, (torch.uint8, torch.float8_e4m3fn))):
        for dtype in dtypes:
            _make("cache", kind=kind, k=_t(64, D, dtype=dtype), v=_t(64, D, dtype=dtype), k_row_scale=None, v_row_scale=None)
    c = cache4.make_cache(**_cache())
    a = cache4.make_rows_args(cache=c, **_rows())
    cache4.make_rows_args(cache=a.cache, **_rows())  # (a cache out of an argument block)


TYPES = [("cache", n, d) for n, d in (("k", BF), ("v", F), ("k_row_scale", BF), ("v_row_scale", torch.float16), ("v_row_scale", torch.uint8), ("cu_L", torch.int64))]
TYPES += [("rows", n, d) for n, d in (("k_rows", F), ("v_rows", torch.float16), ("L", torch.int64), ("path", F))]
TYPES += [("attn", n, d) for n, d in (("q", F), ("k_tree", torch.float16), ("v_tree", F), ("out", F), ("lse", BF), ("lse", torch.float64), ("anc_mask", I),
                                      ("anc_mask", F), ("cu_T", torch.int64))]
TYPES += [("weigh", n, d) for n, d in (("q", F), ("lse", BF), ("weight", BF), ("weight", torch.float16), ("weight", torch.float64), ("pos", F))]
TYPES += [("select", n, d) for n, d in (("weight", BF), ("weight", torch.float16), ("pos", torch.int64), ("src", torch.int64))]
TYPES += [("move", n, d) for n, d in (("weight", BF), ("weight", torch.float64), ("pos", F), ("src", torch.int64))]


@pytest.mark.parametrize("which,name,dtype", TYPES)
def test_other_types_are_refused(which, name, dtype):
    given = {"cache": _cache, "rows": _rows, "attn": _attn, "weigh": _weigh, "select": _select, "move": _move}[which]()[name]
    with pytest.raises(ValueError, match=name):
        _make(which, **{name: torch.zeros(given.shape, dtype=dtype)})


@pytest.mark.parametrize("kind,dtype", [(cache4.ROWS_BF16, F), (cache4.ROWS_BF16, torch.float16), (cache4.ROWS_BF16, torch.uint8), (cache4.ROWS_E4M3, BF),
                                        (cache4.ROWS_E4M3, torch.float8_e5m2)])
def test_caches_of_other_types_are_refused(kind, dtype):
    for name in ("k", "v"):
        good = BF if kind == cache4.ROWS_BF16 else torch.uint8
        kw = dict(k=_t(64, D, dtype=good), v=_t(64, D, dtype=good), k_row_scale=None, v_row_scale=None)
        kw[name] = _t(64, D, dtype=dtype)
        with pytest.raises(ValueError, match=name):
            _make("cache", kind=kind, **kw)


@pytest.mark.parametrize("which,name,shape", [
    ("cache", "page_table", (8,)), ("rows", "v_rows", (B * T, HKV, 128)), ("rows", "v_rows", (1, HKV, D)), ("rows", "L", (B - 1,)), ("rows", "path_len", (B - 1,)),
    ("rows", "path", (B - 1, T)), ("rows", "path", (B, T + 1)), ("rows", "L_out", (B - 1,)), ("attn", "k_tree", (B * T - 1, HKV, D)), ("attn", "v_tree", (B * T, HKV + 1, D)),
    ("attn", "k_tree", (B * T, HKV, 128)), ("attn", "q", (B * T, HQ * D)), ("attn", "out", (B * T - 1, HQ, D)), ("attn", "out", (B * T, D, HQ)),
    ("attn", "lse", (B * T - 1, HQ)), ("attn", "lse", (B * T, HQ + 1)), ("attn", "anc_mask", (B * T - 1, 1)), ("attn", "anc_mask", (B * T,)), ("attn", "L", (B - 1,)),
    ("weigh", "lse", (B * T - 1, HQ)), ("weigh", "lse", (B * T, HKV)), ("weigh", "L", (B - 1,)), ("weigh", "path_len", (B - 1,)), ("weigh", "path", (B - 1, T)),
    ("weigh", "path", (B, T - 1)), ("weigh", "first_pos", (B - 1,)), ("weigh", "pos", (B, HKV, LD - 1)), ("select", "L", (B - 1,)), ("select", "keep", (B - 1,)),
    ("select", "newest", (B - 1,)), ("select", "L_out", (B - 1,)), ("select", "src", (B - 1, HKV, LD)), ("select", "pos", (B, HKV, LD - 1)), ("move", "n", (B - 1,)),
    ("move", "weight", (B, HKV - 1, LD)), ("move", "pos", (B, HKV, LD - 1))])
def test_other_shapes_are_refused(which, name, shape):
    given = {"cache": _paged, "rows": _rows, "attn": _attn, "weigh": _weigh, "select": _select, "move": _move}[which]()[name]
    with pytest.raises(ValueError):
        _make(which, **{name: torch.zeros(shape, dtype=given.dtype)})


def test_weights_of_fewer_sequences_are_refused():
    with pytest.raises(ValueError, match="weight"):
        _make("weigh", weight=_t(B - 1, HKV, LD), pos=_t(B - 1, HKV, LD, dtype=I))


@pytest.mark.parametrize("which", ["rows", "attn", "weigh", "move"])
def test_caches_of_fewer_sequences_are_refused(which):
    with pytest.raises(ValueError, match="cu_L"):
        _make(which, _cache(cu_L=_t(B, dtype=I)))
    with pytest.raises(ValueError, match="page_table"):
        _make(which, _paged(page_table=_t(B - 1, 4, dtype=I)))


@pytest.mark.parametrize("which,name", [("cache", "k"), ("cache", "v_row_scale"), ("rows", "k_rows"), ("rows", "L"), ("rows", "err_flag"), ("attn", "q"), ("attn", "lse"),
                                        ("attn", "workspace"), ("weigh", "weight"), ("weigh", "first_pos"), ("select", "src"), ("select", "keep"), ("move", "n"),
                                        ("move", "weight")])
def test_tensors_on_different_devices_are_refused(which, name):
    given = {"cache": _cache, "rows": lambda: _rows(err_flag=_t(1, dtype=I)), "attn": _attn, "weigh": _weigh, "select": _select, "move": _move}[which]()[name]
    with pytest.raises(ValueError, match="device"):
        _make(which, **{name: given.to("meta")})


@pytest.mark.parametrize("which,name", [("rows", "k_rows"), ("attn", "q"), ("attn", "lse"), ("attn", "out"), ("weigh", "weight"), ("weigh", "lse"), ("select", "weight"),
                                        ("move", "weight")])
def test_tensors_that_are_not_packed_are_refused(which, name):
    given = {"rows": _rows, "attn": _attn, "weigh": _weigh, "select": _select, "move": _move}[which]()[name]
    wide = torch.zeros((*given.shape[:-1], given.shape[-1] * 2), dtype=given.dtype)[..., ::2]
    with pytest.raises(ValueError, match="not contiguous"):
        _make(which, **{name: wide})


def test_calls_on_host_tensors_are_refused():
    c = cache4.make_cache(**_cache())
    attn = _attn()
    where = [attn.pop(n) for n in ("q", "k_tree", "v_tree", "cu_T", "L")]
    for call in (lambda: cache4.store(cache=c, **_rows()), lambda: cache4.load(cache=c, **_rows(L_out=None)),
                 lambda: cache4.tree_verify_attn(where[0], where[1], where[2], c, where[3], where[4], **attn),
                 lambda: evict.key_weights(cache=c, **_weigh()), lambda: evict.select(_t(B, HKV, LD), _t(B, dtype=I), _t(B, dtype=I), max_L=LD, max_keep=LD),
                 lambda: evict.move(cache=c, **_move())):
        with pytest.raises(ValueError, match="GPU"):
            call()
