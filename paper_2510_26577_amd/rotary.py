"""Thin ctypes binding of the first part of include/tva_layer.h (argument marshalling only): rotary positions of the heads of new
tokens' q and k (with the heads' norms), and their K/V to the cache.  Everything on tensors runs as HIP kernels in libtva.so; a
missing library raises (no fallback)."""
from __future__ import annotations

import ctypes

from . import binding
from .binding import _p
from .cache4 import Cache, _at_least, _fits, _indices, _is, _on_current_gpu, _one_device, _typed

PLAIN, LINEAR, BASE, WAVELENGTH, RAMP = range(5)  # tva_rotary_scaling

_ready = False


class RotateArgs(ctypes.Structure):
    """Mirror of `struct tva_rotate_args`."""
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hkv", "D", "sum_T", "dims", "interleaved", "mask_words")] + \
               [("magnitude", ctypes.c_float), ("eps", ctypes.c_float)] + \
               [(n, ctypes.c_void_p) for n in ("cu_T", "L", "pos", "anc_mask", "freq", "q", "k", "q_norm", "k_norm", "q_out", "k_out")] + \
               [(n, ctypes.c_int64) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride")]


class AppendArgs(ctypes.Structure):
    """Mirror of `struct tva_append_args`."""
    _fields_ = [("r", RotateArgs), ("v", ctypes.c_void_p), ("v_stride", ctypes.c_int64), ("cache", Cache), ("L_out", ctypes.c_void_p),
                ("err_flag", ctypes.c_void_p)]


def _lib():
    global _ready
    lib = binding.load_library()
    if not _ready:
        d = ctypes.c_double
        lib.tva_rotary_frequencies.restype = ctypes.c_int
        lib.tva_rotary_frequencies.argtypes = [ctypes.c_int32, ctypes.c_int32, d, d, d, d, d, ctypes.c_void_p, ctypes.c_void_p]
        if lib.tva_sizeof_rotate_args() != ctypes.sizeof(RotateArgs) or lib.tva_sizeof_append_args() != ctypes.sizeof(AppendArgs):
            raise RuntimeError("libtva.so is stale: rebuild it")
        _ready = True
    return lib


def frequencies(dims: int, base: float = 10000.0, *, scaling: int = PLAIN, factor: float = 1.0, original: float = 0.0, low: float = 1.0,
                high: float = 0.0):
    """(numpy float64 [dims/2] radians per position, magnitude): what `freq` (as a device tensor) and `magnitude` of the calls below take.
    high = 0: the usual one of the scaling (4 turns for WAVELENGTH, 32 for RAMP)."""
    import numpy as np
    if dims < 2 or dims % 2:
        raise ValueError("dims is an even number of elements")
    freq, magnitude = np.zeros(dims // 2, np.float64), ctypes.c_double(0.0)
    rc = _lib().tva_rotary_frequencies(int(scaling), int(dims), float(base), float(factor), float(original), float(low),
                                       float(high or {WAVELENGTH: 4.0, RAMP: 32.0}.get(int(scaling), 0.0)), freq.ctypes.data, ctypes.byref(magnitude))
    if rc != binding.TVA_OK:
        raise binding.TvaError(rc)
    return freq, magnitude.value


def _heads(name: str, t):
    """Rows of heads [rows, H, D]; a row's heads lie side by side, rows may lie further apart (a part of a wider projection): the stride."""
    _is(("bfloat16",), t, name)
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1) or (t.shape[1] > 1 and t.stride(1) != t.shape[2]):
        raise ValueError(f"{name} is [rows, heads, D], the heads of a row side by side")
    if t.shape[0] < 2:
        return 0
    stride = t.stride(0)
    if stride % 8 or stride < t.shape[1] * t.shape[2]:
        raise ValueError(f"{name}: rows lie {stride} elements apart")
    return stride


def _rotation(a: RotateArgs, q, k, q_out, k_out, cu_T, L, pos, anc_mask, freq, dims, interleaved, magnitude, q_norm, k_norm, eps):
    some = q if q is not None else k
    if some is None:
        raise ValueError("q or k is given")
    for x, y, name in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None and y is not None:
            raise ValueError(f"{name}_out without {name}")
        if x is not None:
            setattr(a, f"{name}_stride", _heads(name, x))
        if y is not None:
            setattr(a, f"{name}_out_stride", _heads(f"{name}_out", y))
            if y.shape[0] < x.shape[0] or y.shape[1:] != x.shape[1:]:
                raise ValueError(f"{name}_out has a row for every row of {name}")
    if q is not None and q_out is None:
        raise ValueError("q without q_out")
    if q is not None and k is not None and (q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2]):
        raise ValueError("q and k have the same rows and head dimension")
    rows, D, dims = int(some.shape[0]), int(some.shape[2]), int(dims)
    _typed(("bfloat16",), q_norm=q_norm, k_norm=k_norm)
    _typed(("float64",), freq=freq)
    _typed(("int64", "uint64"), anc_mask=anc_mask)
    _indices(cu_T=cu_T, L=L, pos=pos)
    for name, w in (("q_norm", q_norm), ("k_norm", k_norm)):
        if w is not None and w.numel() != D:
            raise ValueError(f"{name} has {w.numel()} entries, not {D}")
    if dims > 0 and (freq is None or freq.numel() < dims // 2):
        raise ValueError("freq has an entry for every pair")
    if anc_mask is not None and (anc_mask.dim() != 2 or anc_mask.shape[0] < rows):
        raise ValueError("anc_mask has a row for every row of q")
    if pos is None and (cu_T is None or L is None):
        raise ValueError("without pos, cu_T and L are given")
    B = cu_T.numel() - 1 if cu_T is not None else 0
    _at_least(B, L=L)
    _at_least(rows, pos=pos)
    a.B, a.Hq, a.Hkv, a.D = B, int(q.shape[1]) if q is not None else 0, int(k.shape[1]) if k is not None else 0, D
    a.sum_T, a.dims, a.interleaved, a.mask_words = rows, dims, int(bool(interleaved)), int(anc_mask.shape[1]) if anc_mask is not None else 0
    a.magnitude, a.eps = float(magnitude), float(eps)
    a.cu_T, a.L, a.pos, a.anc_mask, a.freq = _p(cu_T), _p(L), _p(pos), _p(anc_mask), _p(freq)
    a.q, a.k, a.q_norm, a.k_norm, a.q_out, a.k_out = _p(q), _p(k), _p(q_norm), _p(k_norm), _p(q_out), _p(k_out)
    return (q, k, q_out, k_out, cu_T, L, pos, anc_mask, freq, q_norm, k_norm)


def make_rotate_args(*, freq=None, dims: int, q=None, k=None, q_out=None, k_out=None, cu_T=None, L=None, pos=None, anc_mask=None,
                     interleaved: bool = False, magnitude: float = 1.0, q_norm=None, k_norm=None, eps: float = 1e-6) -> RotateArgs:
    """q bf16 [rows, Hq, D], k bf16 [rows, Hkv, D] (views of a wider projection are fine), freq float64 [dims/2]; q_out and k_out may be
    q and k themselves."""
    a = RotateArgs()
    if k is not None and k_out is None:
        raise ValueError("k without k_out")
    keep = _rotation(a, q, k, q_out, k_out, cu_T, L, pos, anc_mask, freq, dims, interleaved, magnitude, q_norm, k_norm, eps)
    _one_device(*keep)
    # the struct holds raw addresses: keep the tensors alive as long as it lives
    a._keep = keep
    return a


def make_append_args(*, k, v, cache: Cache, cu_T, L, freq=None, dims: int, q=None, q_out=None, k_out=None, pos=None, anc_mask=None,
                     interleaved: bool = False, magnitude: float = 1.0, q_norm=None, k_norm=None, eps: float = 1e-6, L_out=None,
                     err_flag=None) -> AppendArgs:
    """make_rotate_args' arguments, v bf16 [rows, Hkv, D] and the cache (cache4.make_cache); cu_T and L say where the rows go."""
    a = AppendArgs()
    if cu_T is None or L is None:
        raise ValueError("cu_T and L are given")
    if tuple(v.shape) != tuple(k.shape):
        raise ValueError("v has the shape of k")
    a.v_stride = _heads("v", v)
    _indices(L_out=L_out, err_flag=err_flag)
    keep = _rotation(a.r, q, k, q_out, k_out, cu_T, L, pos, anc_mask, freq, dims, interleaved, magnitude, q_norm, k_norm, eps)
    _at_least(a.r.B, L_out=L_out)
    _fits(cache, a.r.B, *keep, v, L_out, err_flag)
    a.v, a.cache, a.L_out, a.err_flag = _p(v), cache, _p(L_out), _p(err_flag)
    a._keep = (*keep, v, cache, L_out, err_flag)
    return a


def rotate_raw(args: RotateArgs, stream=None) -> None:
    """Queue tva_rotate on a prepared argument block."""
    binding.call_raw("tva_rotate", RotateArgs, args, stream)


def append_raw(args: AppendArgs, stream=None) -> None:
    """Queue tva_cache_append on a prepared argument block."""
    binding.call_raw("tva_cache_append", AppendArgs, args, stream)


def rotate(*, stream=None, q=None, k=None, q_out=None, k_out=None, **kw):
    """Keyword arguments of make_rotate_args; outputs that are not given are made (binding.empty_for).  Returns (q_out, k_out)."""
    if q is not None and q_out is None:
        q_out = binding.empty_for(stream, tuple(q.shape), q.dtype, q.device)
    if k is not None and k_out is None:
        k_out = binding.empty_for(stream, tuple(k.shape), k.dtype, k.device)
    args = make_rotate_args(q=q, k=k, q_out=q_out, k_out=k_out, **kw)
    _on_current_gpu(q if q is not None else k)
    rotate_raw(args, stream)
    return q_out, k_out


def append(*, stream=None, q=None, q_out=None, **kw):
    """Keyword arguments of make_append_args; the cache is written in place.  Returns q_out (made where q is given without:
    binding.empty_for)."""
    if q is not None and q_out is None:
        q_out = binding.empty_for(stream, tuple(q.shape), q.dtype, q.device)
    args = make_append_args(q=q, q_out=q_out, **kw)
    _on_current_gpu(kw["k"])
    append_raw(args, stream)
    return q_out
