"""Thin ctypes binding of the attention of include/tva_layer.h (argument marshalling only): new tokens -- a chunk of a prompt, a single
token, a draft tree -- over the cache that holds them, with or without a sliding window.  Everything runs as HIP kernels in libtva.so; a
missing library raises (no fallback)."""
from __future__ import annotations

import ctypes
from typing import Optional

from . import binding
from .binding import _p
from .cache4 import Cache, _at_least, _fits, _indices, _on_current_gpu, _typed
from .rotary import _heads

_ready = False


class ChunkArgs(ctypes.Structure):
    """Mirror of `struct tva_chunk_args`."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "D", "sum_T", "max_T", "max_L", "mask_words", "window", "n_first")] + \
               [("scale", ctypes.c_float), ("num_splits", ctypes.c_int32), ("plan_rows", ctypes.c_int32), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in ("cu_T", "L", "q")] + [("q_stride", ctypes.c_int64), ("anc_mask", ctypes.c_void_p)] + \
               [("cache", Cache), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


def _lib():
    global _ready
    lib = binding.load_library()
    if not _ready:
        lib.tva_chunk_workspace_bytes.restype = ctypes.c_size_t
        for name in ("tva_chunk_plan_rows", "tva_chunk_plan_splits"):
            getattr(lib, name).restype = ctypes.c_int32
        for name in ("tva_chunk_workspace_bytes", "tva_chunk_plan_rows", "tva_chunk_plan_splits"):
            getattr(lib, name).argtypes = [ctypes.POINTER(ChunkArgs)]
        if lib.tva_sizeof_chunk_args() != ctypes.sizeof(ChunkArgs):
            raise RuntimeError("libtva.so is stale: rebuild it")
        _ready = True
    return lib


def make_args(*, q, cache: Cache, cu_T, L, Hkv: int, max_T: int, max_L: int, scale: float, window: int = 0, n_first: int = 0, anc_mask=None,
              out=None, lse=None, workspace=None, num_splits: int = 0, plan_rows: int = 0) -> ChunkArgs:
    """q bf16 [sum_T, Hq, D] (a view of a wider projection is fine), out bf16 like q but packed, lse fp32 [sum_T, Hq] or None (either may
    have more rows, which are left alone)."""
    stride = _heads("q", q)
    _typed(("bfloat16",), out=out)
    _typed(("float32",), lse=lse)
    _typed(("int64", "uint64"), anc_mask=anc_mask)
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace is not contiguous")
    _indices(cu_T=cu_T, L=L)
    rows, Hq, D = q.shape
    if out is not None and (out.dim() != 3 or out.shape[0] < rows or out.shape[1:] != q.shape[1:]):
        raise ValueError("out has a row for every row of q")
    if lse is not None and (lse.dim() != 2 or lse.shape[0] < rows or lse.shape[1] != Hq):
        raise ValueError("lse has a number for every row and head of q")
    if anc_mask is not None and (anc_mask.dim() != 2 or anc_mask.shape[0] < rows):
        raise ValueError("anc_mask has a row for every row of q")
    B = cu_T.numel() - 1
    _at_least(B, L=L)
    _fits(cache, B, q, anc_mask, out, lse, workspace, cu_T, L)
    a = ChunkArgs()
    a.B, a.Hq, a.Hkv, a.D = B, Hq, int(Hkv), D
    a.sum_T, a.max_T, a.max_L, a.window, a.n_first = rows, int(max_T), int(max_L), int(window), int(n_first)
    a.mask_words = int(anc_mask.shape[1]) if anc_mask is not None else 0
    a.scale, a.num_splits, a.plan_rows = float(scale), int(num_splits), int(plan_rows)
    a.cu_T, a.L, a.q, a.q_stride, a.anc_mask, a.cache = _p(cu_T), _p(L), _p(q), stride, _p(anc_mask), cache
    a.out, a.lse, a.workspace = _p(out), _p(lse), _p(workspace)
    a.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    # the struct holds raw addresses: keep the tensors alive as long as it lives
    a._keep = (q, cache, cu_T, L, anc_mask, out, lse, workspace)
    return a


def workspace_bytes(args: ChunkArgs) -> int:
    n = _lib().tva_chunk_workspace_bytes(ctypes.byref(args))
    if n == ctypes.c_size_t(-1).value:
        raise binding.TvaError(-1)
    return int(n)


def plan_rows(args: ChunkArgs) -> int:
    n = _lib().tva_chunk_plan_rows(ctypes.byref(args))
    if n < 0:
        raise binding.TvaError(-1)
    return int(n)


def plan_splits(args: ChunkArgs) -> int:
    n = _lib().tva_chunk_plan_splits(ctypes.byref(args))
    if n < 0:
        raise binding.TvaError(-1)
    return int(n)


def attn_workspace(args: ChunkArgs, device, stream=None):
    """Makes the workspace that the block's shapes need and puts it into the block (None where none is needed); stream: the one that the call
    is going to be queued on, if it is not the current one."""
    import torch
    need = workspace_bytes(args)
    ws = binding.empty_for(stream, need // 4, torch.float32, torch.device(device)) if need else None
    args.workspace, args.workspace_bytes = _p(ws), need
    args._keep = (*args._keep, ws)
    return ws


def attn_raw(args: ChunkArgs, stream=None) -> None:
    """Queue the attention on a prepared argument block."""
    binding.call_raw("tva_chunk_attn", ChunkArgs, args, stream)


def attn(q, cache: Cache, cu_T, L, *, Hkv: int, max_T: int, max_L: int, scale: float, window: int = 0, n_first: int = 0, anc_mask=None, out=None,
         lse=None, workspace=None, num_splits: int = 0, plan_rows: int = 0, stream: Optional[object] = None):
    """Attention of new tokens over the cache that holds them.  Returns (out bf16 [sum_T, Hq, D], lse fp32 [sum_T, Hq]);
    what is not given is made (binding.empty_for)."""
    import torch
    if out is None:
        out = binding.empty_for(stream, tuple(q.shape), torch.bfloat16, q.device)
    if lse is None:
        lse = binding.empty_for(stream, tuple(q.shape[:2]), torch.float32, q.device)
    a = make_args(q=q, cache=cache, cu_T=cu_T, L=L, Hkv=Hkv, max_T=max_T, max_L=max_L, scale=scale, window=window, n_first=n_first,
                  anc_mask=anc_mask, out=out, lse=lse, workspace=workspace, num_splits=num_splits, plan_rows=plan_rows)
    _on_current_gpu(q)
    if workspace is None:
        attn_workspace(a, q.device, stream)
    attn_raw(a, stream)
    return out, lse
