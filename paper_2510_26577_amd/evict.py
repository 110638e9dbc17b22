"""Thin ctypes binding of the eviction part of include/tva_cache.h (argument marshalling only): the attention that cached
keys receive, the slots that stay, and the move that closes the gaps.  Everything runs as HIP kernels in libtva.so; a
missing library raises (no fallback)."""
from __future__ import annotations

import ctypes

from . import binding
from .binding import _p
from .cache4 import Cache, _at_least, _fits, _indices, _on_gpu, _one_device, _typed

_ready = False


class KeyWeightArgs(ctypes.Structure):
    """Mirror of `struct tva_key_weight_args`."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "D", "max_rows", "max_L")] + \
               [("scale", ctypes.c_float), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in ("cu_T", "path", "path_len", "L", "q", "lse")] + \
               [("cache", Cache), ("weight", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("first_pos", ctypes.c_void_p), ("ld", ctypes.c_int64)]


class SelectArgs(ctypes.Structure):
    """Mirror of `struct tva_evict_select_args`."""
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "B", "H", "max_L", "n_first", "reserved")] + \
               [(n, ctypes.c_void_p) for n in ("L", "keep", "newest", "weight", "pos")] + \
               [("ld", ctypes.c_int64), ("src", ctypes.c_void_p), ("ld_src", ctypes.c_int64), ("L_out", ctypes.c_void_p)]


class MoveArgs(ctypes.Structure):
    """Mirror of `struct tva_evict_move_args`."""
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "B", "H", "Hkv", "D", "max_keep")] + \
               [("n", ctypes.c_void_p), ("src", ctypes.c_void_p), ("ld_src", ctypes.c_int64), ("cache", Cache),
                ("layer_stride_cache", ctypes.c_int64), ("weight", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("ld", ctypes.c_int64),
                ("err_flag", ctypes.c_void_p)]


def _lib():
    global _ready
    lib = binding.load_library()
    if not _ready:
        for name, block in (("tva_key_weights", KeyWeightArgs), ("tva_evict_select", SelectArgs), ("tva_evict_move", MoveArgs)):
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name).argtypes = [ctypes.POINTER(block), ctypes.c_void_p]
        if (lib.tva_sizeof_key_weight_args(), lib.tva_sizeof_evict_select_args(), lib.tva_sizeof_evict_move_args()) != \
                tuple(ctypes.sizeof(b) for b in (KeyWeightArgs, SelectArgs, MoveArgs)):
            raise RuntimeError("libtva.so is stale: rebuild it")
        _ready = True
    return lib


def make_key_weight_args(*, q, lse, cache: Cache, cu_T, L, weight, max_rows: int, max_L: int, scale: float, path=None, path_len=None,
                         pos=None, first_pos=None) -> KeyWeightArgs:
    """q bf16 [sum_T, Hq, D] and lse fp32 [sum_T, Hq] of a step's attention; weight fp32 (and pos int32) [B, Hkv, ld]."""
    _typed(("bfloat16",), q=q)
    _typed(("float32",), lse=lse, weight=weight)
    _indices(cu_T=cu_T, L=L, path=path, path_len=path_len, pos=pos, first_pos=first_pos)
    a = KeyWeightArgs()
    a.B, a.Hq, a.Hkv, a.D = cu_T.numel() - 1, int(q.shape[1]), int(weight.shape[1]), int(q.shape[2])
    a.max_rows, a.max_L, a.scale = int(max_rows), int(max_L), float(scale)
    if path is not None and int(path.shape[1]) != a.max_rows:
        raise ValueError("max_rows is the row length of path")
    if pos is not None and tuple(pos.shape) != tuple(weight.shape):
        raise ValueError("pos has the shape of weight")
    if tuple(lse.shape) != tuple(q.shape[:2]):
        raise ValueError("lse has a number for every row and head of q")
    if weight.dim() != 3 or weight.shape[0] < a.B:
        raise ValueError("weight is [B, Hkv, ld]")
    _at_least(a.B, L=L, path_len=path_len, first_pos=first_pos)
    _at_least(a.B * a.max_rows, path=path)
    _fits(cache, a.B, q, lse, weight, pos, cu_T, L, path, path_len, first_pos)
    a.cu_T, a.path, a.path_len, a.L, a.q, a.lse = _p(cu_T), _p(path), _p(path_len), _p(L), _p(q), _p(lse)
    a.cache, a.weight, a.pos, a.first_pos, a.ld = cache, _p(weight), _p(pos), _p(first_pos), int(weight.shape[2])
    # the struct holds raw addresses: keep the tensors alive as long as it lives
    a._keep = (cu_T, path, path_len, L, q, lse, cache, weight, pos, first_pos)
    return a


def make_select_args(*, weight, L, keep, max_L: int, src, L_out=None, n_first: int = 0, newest=None, pos=None) -> SelectArgs:
    """weight fp32 (and pos int32) [n_layers, B, H, ld] or [B, H, ld], src int32 likewise with ld_src."""
    _typed(("float32",), weight=weight)
    _indices(L=L, keep=keep, src=src, L_out=L_out, newest=newest, pos=pos)
    a = SelectArgs()
    if tuple(src.shape[:-1]) != tuple(weight.shape[:-1]) or (pos is not None and tuple(pos.shape) != tuple(weight.shape)):
        raise ValueError("weight, pos and src have the same rows")
    if weight.dim() not in (3, 4):
        raise ValueError("weight is [B, H, ld] or [n_layers, B, H, ld]")
    _at_least(int(weight.shape[-3]), L=L, keep=keep, newest=newest, L_out=L_out)
    _one_device(weight, pos, src, L, keep, newest, L_out)
    a.n_layers = int(weight.shape[0]) if weight.dim() == 4 else 1
    a.B, a.H, a.max_L, a.n_first = int(weight.shape[-3]), int(weight.shape[-2]), int(max_L), int(n_first)
    a.L, a.keep, a.newest, a.weight, a.pos = _p(L), _p(keep), _p(newest), _p(weight), _p(pos)
    a.ld, a.src, a.ld_src, a.L_out = int(weight.shape[-1]), _p(src), int(src.shape[-1]), _p(L_out)
    a._keep = (L, keep, newest, weight, pos, src, L_out)
    return a


def make_move_args(*, src, n, cache: Cache, Hkv: int, D: int, max_keep: int, weight=None, pos=None, layer_stride_cache: int = 0,
                   err_flag=None) -> MoveArgs:
    """src int32 [n_layers, B, H, ld_src] or [B, H, ld_src] (H = Hkv, or 1: shared by the heads), n: select's L_out."""
    _typed(("float32",), weight=weight)
    _indices(src=src, n=n, pos=pos, err_flag=err_flag)
    a = MoveArgs()
    for t in (weight, pos):
        if t is not None and tuple(t.shape[:-1]) != tuple(src.shape[:-1]):
            raise ValueError("src, weight and pos have the same rows")
    if weight is not None and pos is not None and weight.shape[-1] != pos.shape[-1]:
        raise ValueError("pos has the shape of weight")
    if src.dim() not in (3, 4):
        raise ValueError("src is [B, H, ld_src] or [n_layers, B, H, ld_src]")
    _at_least(int(src.shape[-3]), n=n)
    _fits(cache, int(src.shape[-3]), src, n, weight, pos, err_flag)
    a.n_layers = int(src.shape[0]) if src.dim() == 4 else 1
    a.B, a.H, a.Hkv, a.D, a.max_keep = int(src.shape[-3]), int(src.shape[-2]), int(Hkv), int(D), int(max_keep)
    a.n, a.src, a.ld_src, a.cache, a.layer_stride_cache = _p(n), _p(src), int(src.shape[-1]), cache, int(layer_stride_cache)
    a.weight, a.pos, a.err_flag = _p(weight), _p(pos), _p(err_flag)
    a.ld = int((weight if weight is not None else pos).shape[-1]) if weight is not None or pos is not None else 0
    a._keep = (n, src, cache, weight, pos, err_flag)
    return a


def key_weights_raw(args: KeyWeightArgs, stream=None) -> None:
    binding.call_raw("tva_key_weights", KeyWeightArgs, args, stream)


def select_raw(args: SelectArgs, stream=None) -> None:
    binding.call_raw("tva_evict_select", SelectArgs, args, stream)


def move_raw(args: MoveArgs, stream=None) -> None:
    binding.call_raw("tva_evict_move", MoveArgs, args, stream)


def key_weights(*, stream=None, **kw) -> None:
    """Keyword arguments of make_key_weight_args; weight (and pos) are brought up to date in place."""
    args = make_key_weight_args(**kw)
    _on_gpu(kw["q"])
    key_weights_raw(args, stream)


def select(weight, L, keep, *, max_L: int, max_keep: int, n_first: int = 0, newest=None, pos=None, src=None, L_out=None, stream=None):
    """Which slots stay: returns (src int32 [.., max_keep], L_out int32 [B]); entries of src from L_out[b] on are not written."""
    import torch
    if src is None:
        src = binding.empty_for(stream, (*weight.shape[:-1], max(1, int(max_keep))), torch.int32, weight.device)
    if L_out is None:
        L_out = binding.empty_for(stream, int(weight.shape[-3]), torch.int32, weight.device)
    args = make_select_args(weight=weight, L=L, keep=keep, max_L=max_L, src=src, L_out=L_out, n_first=n_first, newest=newest, pos=pos)
    _on_gpu(weight)
    select_raw(args, stream)
    return src, L_out


def move(*, stream=None, **kw) -> None:
    """Keyword arguments of make_move_args; cache, weight and pos are changed in place."""
    args = make_move_args(**kw)
    _on_gpu(kw["src"])
    move_raw(args, stream)
