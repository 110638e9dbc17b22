"""Thin ctypes binding of the 4-bit rows of include/tva_cache.h (argument marshalling only): bf16 rows stored to a cache of
4-bit rows and read back, and the verification attention over such a cache.  Everything runs as HIP kernels in libtva.so;
a missing library raises (no fallback)."""
from __future__ import annotations

import ctypes
from typing import Optional

from . import binding
from .binding import _p

ROWS_BF16, ROWS_E4M3, ROWS_E2M1 = range(3)  # tva_row_kind

_ready = False


class Cache(ctypes.Structure):
    """Mirror of `struct tva_cache`."""
    _fields_ = [("kind", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("k_scale", ctypes.c_float),
                ("v_scale", ctypes.c_float), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "k_row_scale", "v_row_scale", "cu_L", "page_table")] + \
               [(n, ctypes.c_int64) for n in ("stride_page", "stride_tok", "stride_head")]


class RowsArgs(ctypes.Structure):
    """Mirror of `struct tva_rows_args`."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hkv", "D", "max_rows")] + \
               [(n, ctypes.c_void_p) for n in ("cu_T", "L", "path", "path_len", "k_rows", "v_rows")] + \
               [("cache", Cache), ("L_out", ctypes.c_void_p), ("err_flag", ctypes.c_void_p), ("n_layers", ctypes.c_int32),
                ("layer_stride_cache", ctypes.c_int64), ("layer_stride_rows", ctypes.c_int64)]


class Attn4Args(ctypes.Structure):
    """Mirror of `struct tva_attn4_args`."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "D", "sum_T", "max_T", "mask_words", "max_L")] + \
               [("scale", ctypes.c_float), ("num_splits", ctypes.c_int32), ("plan_rows", ctypes.c_int32), ("reserved", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in ("cu_T", "L", "q", "k_tree", "v_tree", "anc_mask", "parent")] + \
               [("cache", Cache), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


def _lib():
    global _ready
    lib = binding.load_library()
    if not _ready:
        vp = ctypes.c_void_p
        for name, block in (("tva_cache_store", RowsArgs), ("tva_cache_load", RowsArgs), ("tva_tree_verify_attn_4bit", Attn4Args)):
            getattr(lib, name).restype = ctypes.c_int
            getattr(lib, name).argtypes = [ctypes.POINTER(block), vp]
        lib.tva_attn4_workspace_bytes.restype = ctypes.c_size_t
        lib.tva_attn4_workspace_bytes.argtypes = [ctypes.POINTER(Attn4Args)]
        lib.tva_attn4_plan_splits.restype = ctypes.c_int32
        lib.tva_attn4_plan_splits.argtypes = [ctypes.POINTER(Attn4Args)]
        if lib.tva_sizeof_rows_args() != ctypes.sizeof(RowsArgs) or lib.tva_sizeof_attn4_args() != ctypes.sizeof(Attn4Args):
            raise RuntimeError("libtva.so is stale: rebuild it")
        _ready = True
    return lib


_dtypes = {}  # names -> torch's types, looked up once


def _is(types, t, name: str) -> None:
    known = _dtypes.get(types)
    if known is None:
        import torch
        known = _dtypes[types] = tuple(getattr(torch, n) for n in types)
    if t.dtype not in known:
        raise ValueError(f"{name} is {t.dtype}, not {' or '.join(types)}")


def _typed(types, **tensors) -> None:
    """What is passed as an address alone has the type that the kernels read and write, and is packed."""
    for name, t in tensors.items():
        if t is not None:
            _is(types, t, name)
            if not t.is_contiguous():
                raise ValueError(f"{name} is not contiguous")


def _indices(**tensors) -> None:
    for name, t in tensors.items():
        if t is not None and (t.element_size() != 4 or t.is_floating_point() or not t.is_contiguous()):
            raise ValueError(f"{name} is a contiguous int32 tensor")


def _at_least(count: int, **tensors) -> None:
    """One entry per sequence (or `count` in all)."""
    for name, t in tensors.items():
        if t is not None and t.numel() < count:
            raise ValueError(f"{name} has {t.numel()} entries, not {count}")


def _one_device(*tensors) -> None:
    first = None
    for t in tensors:
        if t is None:
            continue
        if first is None:
            first = t.device
        elif t.device != first:
            raise ValueError("tensors lie on different devices")


def _on_gpu(t) -> None:
    """(All of a call's tensors lie on one device: one of them says which.)"""
    if not t.is_cuda:
        raise ValueError(f"tensors lie on {t.device}, not on a GPU")


def _fits(cache, B: int, *tensors) -> None:
    """The sequences' places are there, and everything lies on one device (of a cache made here; a copy is not looked into)."""
    k = getattr(cache, "_keep", ())
    _one_device(*tensors, *k)
    if k:
        cu_L, page_table = k[4:6]
        if cu_L is not None and cu_L.numel() < B + 1:
            raise ValueError(f"cu_L has {cu_L.numel()} entries for {B} sequences")
        if page_table is not None and page_table.shape[0] < B:
            raise ValueError(f"page_table has {page_table.shape[0]} rows for {B} sequences")


_ROW_TYPES = {ROWS_BF16: ("bfloat16",), ROWS_E4M3: ("uint8", "float8_e4m3fn"), ROWS_E2M1: ("uint8",)}


def make_cache(*, k, v=None, k_row_scale=None, v_row_scale=None, kind: int = ROWS_E2M1, cu_L=None, page_table=None, page_size: int = 0,
               strides=(0, 0, 0), k_scale: float = 1.0, v_scale: float = 1.0) -> Cache:
    """A cache's tensors, any shape: where a row lies is said by the strides (elements of page, token, head; 0 = packed
    token-major).  v may be left out where only K is read (evict.key_weights)."""
    _indices(cu_L=cu_L, page_table=page_table)
    if page_table is not None and page_table.dim() != 2:
        raise ValueError("page_table has a row per sequence")
    rows = _ROW_TYPES.get(int(kind))  # (another kind: the library refuses it)
    for name, t, types in (("k", k, rows), ("v", v, rows), ("k_row_scale", k_row_scale, ("uint8",)), ("v_row_scale", v_row_scale, ("bfloat16",))):
        if t is not None and types is not None:
            _is(types, t, name)
    _one_device(k, v, k_row_scale, v_row_scale, cu_L, page_table)
    c = Cache()
    c.kind, c.page_size, c.max_pages = int(kind), int(page_size), int(page_table.shape[1]) if page_table is not None else 0
    c.k_scale, c.v_scale = float(k_scale), float(v_scale)
    c.k, c.v, c.k_row_scale, c.v_row_scale = _p(k), _p(v), _p(k_row_scale), _p(v_row_scale)
    c.cu_L, c.page_table = _p(cu_L), _p(page_table)
    c.stride_page, c.stride_tok, c.stride_head = (int(s) for s in strides)
    # the struct holds raw addresses: keep the tensors alive as long as it lives (a copy inside an argument block has them
    # through that block)
    c._keep = (k, v, k_row_scale, v_row_scale, cu_L, page_table)
    return c


def make_rows_args(*, k_rows, v_rows, cu_T, L, cache: Cache, max_rows: int, path=None, path_len=None, L_out=None, err_flag=None,
                   n_layers: int = 0, layer_stride_cache: int = 0, layer_stride_rows: int = 0) -> RowsArgs:
    """k_rows, v_rows: bf16 [.., Hkv, D] (with n_layers > 1 the first layer's lead, the others layer_stride_rows elements further on)."""
    _typed(("bfloat16",), k_rows=k_rows, v_rows=v_rows)
    _indices(cu_T=cu_T, L=L, path=path, path_len=path_len, L_out=L_out, err_flag=err_flag)
    a = RowsArgs()
    a.B, a.Hkv, a.D, a.max_rows = cu_T.numel() - 1, int(k_rows.shape[-2]), int(k_rows.shape[-1]), int(max_rows)
    if path is not None and int(path.shape[1]) != a.max_rows:
        raise ValueError("max_rows is the row length of path")
    if tuple(v_rows.shape) != tuple(k_rows.shape):
        raise ValueError("v_rows has the shape of k_rows")
    _at_least(a.B, L=L, path_len=path_len, L_out=L_out)
    _at_least(a.B * a.max_rows, path=path)
    _fits(cache, a.B, k_rows, v_rows, cu_T, L, path, path_len, L_out, err_flag)
    a.cu_T, a.L, a.path, a.path_len, a.k_rows, a.v_rows = _p(cu_T), _p(L), _p(path), _p(path_len), _p(k_rows), _p(v_rows)
    a.cache, a.L_out, a.err_flag = cache, _p(L_out), _p(err_flag)
    a.n_layers, a.layer_stride_cache, a.layer_stride_rows = int(n_layers), int(layer_stride_cache), int(layer_stride_rows)
    a._keep = (cu_T, L, path, path_len, k_rows, v_rows, cache, L_out, err_flag)
    return a


def store_raw(args: RowsArgs, stream=None) -> None:
    """Queue tva_cache_store on a prepared argument block."""
    binding.call_raw("tva_cache_store", RowsArgs, args, stream)


def load_raw(args: RowsArgs, stream=None) -> None:
    """Queue tva_cache_load on a prepared argument block."""
    binding.call_raw("tva_cache_load", RowsArgs, args, stream)


def store(*, stream=None, **kw) -> None:
    """Keyword arguments of make_rows_args: bf16 rows (a prompt, or an accepted path) become 4-bit rows of the cache, in place."""
    args = make_rows_args(**kw)
    _on_gpu(kw["k_rows"])
    store_raw(args, stream)


def load(*, stream=None, **kw) -> None:
    """Keyword arguments of make_rows_args: the values of the cache's 4-bit rows are written to k_rows and v_rows."""
    args = make_rows_args(**kw)
    _on_gpu(kw["k_rows"])
    load_raw(args, stream)


def make_attn_args(*, q, k_tree, v_tree, cache: Cache, cu_T, L, max_T: int, max_L: int, scale: float, anc_mask=None, parent=None, out=None,
                   lse=None, workspace=None, num_splits: int = 0, plan_rows: int = 0) -> Attn4Args:
    """q bf16 [sum_T, Hq, D], k_tree / v_tree bf16 [sum_T, Hkv, D], out bf16 like q, lse fp32 [sum_T, Hq] or None (either may have
    more rows, which are left alone)."""
    _typed(("bfloat16",), q=q, k_tree=k_tree, v_tree=v_tree, out=out)
    _typed(("float32",), lse=lse)
    _typed(("int64", "uint64"), anc_mask=anc_mask)
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace is not contiguous")
    _indices(cu_T=cu_T, L=L, parent=parent)
    shape, tree = q.shape, k_tree.shape
    if len(shape) != 3 or len(tree) != 3 or tree[0] < shape[0] or tree[2] != shape[2] or v_tree.shape != tree:
        raise ValueError("q is [sum_T, Hq, D], k_tree and v_tree are [sum_T, Hkv, D]")
    rows = shape[0]
    if out is not None and (out.shape[0] < rows or out.shape[1:] != shape[1:]):
        raise ValueError("out has a row for every row of q")
    if lse is not None and (lse.dim() != 2 or lse.shape[0] < rows or lse.shape[1] != shape[1]):
        raise ValueError("lse has a number for every row and head of q")
    if anc_mask is not None and (anc_mask.dim() != 2 or anc_mask.shape[0] < rows):
        raise ValueError("anc_mask has a row for every row of q")
    if parent is not None and parent.numel() < rows:
        raise ValueError("parent has an entry for every row of q")
    B = cu_T.numel() - 1
    _at_least(B, L=L)
    _fits(cache, B, q, k_tree, v_tree, anc_mask, out, lse, workspace, cu_T, L, parent)
    a = Attn4Args()
    a.B = B
    a.sum_T, a.Hq, a.D = shape
    a.Hkv = tree[1]
    a.max_T, a.max_L, a.num_splits, a.plan_rows = int(max_T), int(max_L), int(num_splits), int(plan_rows)
    a.mask_words = int(anc_mask.shape[1]) if anc_mask is not None else max(1, (int(max_T) + 63) // 64)
    a.scale = float(scale)
    a.cu_T, a.L, a.q, a.k_tree, a.v_tree = _p(cu_T), _p(L), _p(q), _p(k_tree), _p(v_tree)
    a.anc_mask, a.parent, a.cache, a.out, a.lse = _p(anc_mask), _p(parent), cache, _p(out), _p(lse)
    a.workspace = _p(workspace)
    a.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    a._keep = (cu_T, L, q, k_tree, v_tree, anc_mask, parent, cache, out, lse, workspace)
    return a


def workspace_bytes(args: Attn4Args) -> int:
    n = _lib().tva_attn4_workspace_bytes(ctypes.byref(args))
    if n == ctypes.c_size_t(-1).value:
        raise binding.TvaError(-1)
    return int(n)


def plan_splits(args: Attn4Args) -> int:
    n = _lib().tva_attn4_plan_splits(ctypes.byref(args))
    if n < 0:
        raise binding.TvaError(-1)
    return int(n)


def attn_workspace(args: Attn4Args, device):
    """Makes the workspace that the block's shapes need and puts it into the block (None where none is needed)."""
    import torch
    need = workspace_bytes(args)
    ws = torch.empty(need // 4, dtype=torch.float32, device=device) if need else None
    args.workspace, args.workspace_bytes = _p(ws), need
    args._keep = (*args._keep, ws)
    return ws


def tree_verify_attn_raw(args: Attn4Args, stream=None) -> None:
    """Queue the attention on a prepared argument block."""
    binding.call_raw("tva_tree_verify_attn_4bit", Attn4Args, args, stream)


def tree_verify_attn(q, k_tree, v_tree, cache: Cache, cu_T, L, *, max_T: int, max_L: int, scale: float, anc_mask=None, parent=None, out=None,
                     lse=None, workspace=None, num_splits: int = 0, plan_rows: int = 0, stream: Optional[object] = None):
    """Tree-masked verification attention over a cache of 4-bit rows.  Returns (out bf16 [sum_T, Hq, D], lse fp32 [sum_T, Hq])."""
    import torch
    if out is None:
        out = torch.empty(tuple(q.shape), dtype=torch.bfloat16, device=q.device)
    if lse is None:
        lse = torch.empty(tuple(q.shape[:2]), dtype=torch.float32, device=q.device)
    a = make_attn_args(q=q, k_tree=k_tree, v_tree=v_tree, cache=cache, cu_T=cu_T, L=L, max_T=max_T, max_L=max_L, scale=scale, anc_mask=anc_mask,
                       parent=parent, out=out, lse=lse, workspace=workspace, num_splits=num_splits, plan_rows=plan_rows)
    _on_gpu(q)
    ws = attn_workspace(a, q.device) if workspace is None else None
    tree_verify_attn_raw(a, stream)
    if ws is not None and stream is not None:  # it goes back to the current stream's pool: not before the work on `stream` is done
        ws.record_stream(stream)
    return out, lse
