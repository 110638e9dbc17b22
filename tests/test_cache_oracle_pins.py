"""Pins of oracle/cache_oracle.py: cases whose result is known without it, and the library's host-side checks (CPU)."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import cache_oracle as orc
from paper_2510_26577_amd import binding, cache4, evict

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        binding.build_library()
    cache4._lib(), evict._lib()
    return binding.load_library()


# ---- the formats ----
def test_codes_of_a_known_row():
    x = np.zeros(64)
    x[:10] = [6.0, -6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.2]
    codes, scales = orc.encode(x, 32, 1)
    assert scales.tolist() == [1.0, 2.0 ** -96]
    assert codes[:10].tolist() == [7, 15, 0, 2, 2, 4, 4, 6, 6, 8]  # half-way values go to the even code


def test_scales_are_the_smallest_that_reach():
    rng = np.random.default_rng(0)
    for a in np.concatenate([np.abs(rng.standard_normal(200)), [6.0, 6.0000001, 3.0, 1e-20, 1e20]]):
        s = orc._scale(a, 1)
        assert np.frexp(s)[0] == 0.5 and 6 * s >= a > 3 * s
        s = orc._scale(a, 4)
        m = np.frexp(s)[0] * 16
        assert m == int(m) and 6 * s >= a and 6 * (s - np.ldexp(1.0, np.frexp(s)[1] - 4)) < a  # (the next smaller number of 4 bits)


def test_extremes_and_what_is_not_finite():
    codes, scales = orc.encode(np.array([np.inf, -np.inf, np.nan, 1.0] + [0.0] * 28), 32, 1)
    assert codes[:4].tolist() == [7, 15, 0, 6] and scales[0] == 0.25
    codes, scales = orc.encode(np.full(32, 3e38), 32, 1)
    assert scales[0] == 2.0 ** 124 and (codes == 7).all()
    codes, scales = orc.encode(np.full(32, 1e-35), 32, 4)
    assert scales[0] == 2.0 ** -96 and (codes == 0).all()


def test_values_decode_to_what_was_encoded():
    rng = np.random.default_rng(1)
    k = orc.to_bf16(rng.standard_normal((5, 2, 128)))
    kb, ks, vb, vs = orc.encode_rows(k, k)
    x = orc.bf16(k)
    assert np.abs(orc.decode_k(kb, ks) - x).max() <= np.abs(x).max() / 6 * 2 and np.abs(orc.decode_v(vb, vs) - x).max() <= np.abs(x).max() / 4
    again = orc.encode_rows(orc.to_bf16(orc.decode_k(kb, ks)), orc.to_bf16(orc.decode_v(vb, vs)))
    assert np.array_equal(orc.decode_k(*again[:2]), orc.decode_k(kb, ks)) and np.array_equal(orc.decode_v(*again[2:]), orc.decode_v(vb, vs))


# ---- attention, weights, choice ----
def test_attention_with_zero_queries_is_the_mean():
    rng = np.random.default_rng(2)
    V = rng.standard_normal((7, 2, 64))
    seen = np.ones((3, 7), bool)
    seen[1, 4:] = False
    seen[2] = False
    out, lse, _, _ = orc.attention(np.zeros((3, 4, 64)), rng.standard_normal((7, 2, 64)), V, seen, 1.0)
    assert np.allclose(out[0, 3], V[:, 1].mean(0)) and np.allclose(out[1, 0], V[:4, 0].mean(0)) and not out[2].any()
    assert np.allclose(lse[0], np.log(7)) and np.allclose(lse[1], np.log(4)) and np.isneginf(lse[2]).all()


def test_weights_of_all_seen_keys_add_up_to_the_rows():
    rng = np.random.default_rng(3)
    L, n = 20, 3
    q, K = rng.standard_normal((n, 4, 64)), rng.standard_normal((L, 2, 64))
    seen = np.arange(L) <= np.arange(L - n, L)[:, None]
    lse = orc.attention(q, K, K, seen, 0.1)[1]
    w, _ = orc.key_weights(np.full((2, L), 0.5), q, lse, K, n, 0.1)
    assert np.allclose(w.sum(1), 0.5 * (L - n) + n * 2)
    assert np.allclose(w[:, L - 1], np.exp(0.1 * (q[-1].reshape(2, 2, 64) * K[-1][:, None]).sum(-1) - lse[-1].reshape(2, 2)).sum(1))


def test_choice_of_a_known_row():
    w = np.array([0.0, 5.0, 1.0, 1.0, 9.0, 1.0, np.nan, 0.5])
    assert orc.select(w, 4).tolist() == [4, 1, 2, 3]
    assert orc.select(w, 4, n_first=1).tolist() == [0, 1, 2, 4]
    assert orc.select(w, 4, newest=6).tolist() == [4, 1, 6, 7]
    assert orc.select(w, 3, newest=2, pos=np.array([0, 9, 1, 1, 1, 8, 1, 7])).tolist() == [5, 1, 7]
    assert orc.select(w, 20).tolist() == list(range(8)) and orc.select(w, 0).tolist() == []


# ---- the library's interface ----
def test_exports_match_header(lib):
    text = re.sub(r"/\*.*?\*/", " ", open(os.path.join(binding.INCLUDE_DIR, "tva_cache.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(tva_\w+)\s*\(", text)) == set(binding.CACHE_EXPORTS)
    for name in binding.CACHE_EXPORTS:
        getattr(lib, name)


def _cache(**kw):
    c = cache4.Cache()
    c.kind, c.k, c.v, c.k_row_scale, c.v_row_scale, c.cu_L = cache4.ROWS_E2M1, 4096, 4096, 4096, 4096, 4096
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [(dict(kind=3), -1), (dict(kind=-1), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(k=4100), -1), (dict(k_row_scale=None), -1),
              (dict(v_row_scale=None), -1), (dict(k_row_scale=4098), -1), (dict(v_row_scale=4097), -1), (dict(cu_L=None), -1),
              (dict(page_table=4096, page_size=16, max_pages=4), -1), (dict(cu_L=None, page_table=4096, page_size=0, max_pages=4), -1),
              (dict(cu_L=None, page_table=4096, page_size=16, max_pages=0), -1), (dict(stride_tok=-128), -1), (dict(stride_head=64), -1)]


def _rows(cache=None, **kw):
    a = cache4.RowsArgs()
    a.B, a.Hkv, a.D, a.max_rows = 2, 8, 128, 4
    a.cu_T = a.L = a.path = a.path_len = a.k_rows = a.v_rows = 4096
    a.cache = cache or _cache()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [(dict(B=-1), -1), (dict(Hkv=0), -1), (dict(D=96), -2), (dict(max_rows=-1), -1), (dict(cu_T=None), -1),
                                     (dict(L=None), -1), (dict(path=None), -1), (dict(path_len=None), -1), (dict(k_rows=None), -1),
                                     (dict(v_rows=4104), -1), (dict(L_out=4096), -1), (dict(n_layers=-1), -1), (dict(layer_stride_cache=64), -1),
                                     (dict(layer_stride_rows=4), -1), (dict(B=65536), -2), (dict(n_layers=65536), -2)])
def test_store_and_load_refuse(lib, kw, code):
    assert lib.tva_cache_store(ctypes.byref(_rows(**kw)), None) == code
    assert lib.tva_cache_load(ctypes.byref(_rows(**kw)), None) == code


def test_store_and_load_refuse_what_is_no_call(lib):
    assert lib.tva_cache_store(None, None) == -1 and lib.tva_cache_load(None, None) == -1
    assert lib.tva_cache_load(ctypes.byref(_rows(L_out=8192)), None) == -1
    for kind in (cache4.ROWS_BF16, cache4.ROWS_E4M3):
        assert lib.tva_cache_store(ctypes.byref(_rows(_cache(kind=kind))), None) == -2
    assert lib.tva_cache_store(ctypes.byref(_rows(B=0)), None) == 0 and lib.tva_cache_store(ctypes.byref(_rows(max_rows=0, L_out=None)), None) == 0


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_cache_arguments_are_checked(lib, kw, code):
    assert lib.tva_cache_store(ctypes.byref(_rows(_cache(**kw))), None) == code
    k_only = set(kw) <= {"v", "v_row_scale"}
    if kw.get("kind", 2) == 2:
        assert lib.tva_tree_verify_attn_4bit(ctypes.byref(_attn(_cache(**kw))), None) == code
    if not k_only:
        assert lib.tva_key_weights(ctypes.byref(_weigh(_cache(**kw))), None) == code
    assert lib.tva_evict_move(ctypes.byref(_move(_cache(**kw))), None) == code


def _attn(cache=None, **kw):
    a = cache4.Attn4Args()
    a.B, a.Hq, a.Hkv, a.D, a.sum_T, a.max_T, a.mask_words, a.max_L, a.scale = 2, 32, 8, 128, 20, 10, 1, 100, 0.1
    a.cu_T = a.L = a.q = a.k_tree = a.v_tree = a.anc_mask = a.out = a.lse = a.workspace = 4096
    a.num_splits, a.workspace_bytes = 1, 0
    a.cache = cache or _cache()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [(dict(B=0), -1), (dict(Hq=12), -1), (dict(Hkv=0), -1), (dict(D=96), -2), (dict(max_T=129), -2),
                                     (dict(max_T=65), -2), (dict(mask_words=3), -2), (dict(mask_words=0), -2), (dict(max_L=-1), -1),
                                     (dict(num_splits=-1), -1), (dict(plan_rows=96), -1), (dict(plan_rows=-32), -1), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(cu_T=None), -1),
                                     (dict(L=None), -1), (dict(q=None), -1), (dict(k_tree=None), -1), (dict(v_tree=None), -1), (dict(out=None), -1),
                                     (dict(anc_mask=None), -1), (dict(q=4104), -1), (dict(out=4104), -1), (dict(num_splits=2), -3),
                                     (dict(num_splits=2, workspace=None, workspace_bytes=1 << 30), -1), (dict(num_splits=2, workspace=4100, workspace_bytes=1 << 30), -1),
                                     (dict(B=70000), -2), (dict(max_L=0x7fffffff), -2)])
def test_attention_refuses(lib, kw, code):
    assert lib.tva_tree_verify_attn_4bit(ctypes.byref(_attn(**kw)), None) == code


def test_attention_refuses_other_caches_and_takes_nothing_for_nothing(lib):
    assert lib.tva_tree_verify_attn_4bit(None, None) == -1
    assert lib.tva_tree_verify_attn_4bit(ctypes.byref(_attn(_cache(kind=cache4.ROWS_BF16))), None) == -2
    assert lib.tva_tree_verify_attn_4bit(ctypes.byref(_attn(sum_T=0)), None) == 0 and lib.tva_tree_verify_attn_4bit(ctypes.byref(_attn(max_T=0)), None) == 0


def test_attention_refuses_strides_whose_tiles_need_longer_offsets(lib):
    for D, most in ((128, 1 << 25), (64, 1 << 25)):
        assert lib.tva_tree_verify_attn_4bit(ctypes.byref(_attn(_cache(stride_tok=most), D=D, num_splits=1)), None) == -2


def test_attention_plan(lib):
    for B in (1, 3, 64):
        for L in (0, 1, 64, 65, 1000, 32768):
            for T in (1, 8, 60, 128):
                for splits in (0, 1, 7):
                    a = _attn(B=B, max_L=L, max_T=T, sum_T=B * T, num_splits=splits)
                    s = cache4.plan_splits(a)
                    tiles = -(-L // 64) + -(-T // 64)
                    assert 1 <= s <= tiles * min(B, 64) and (splits == 0 or s <= min(splits, tiles))
                    assert (cache4.workspace_bytes(a) == 0) == (s == 1)
    assert lib.tva_attn4_workspace_bytes(ctypes.byref(_attn(D=32))) == ctypes.c_size_t(-1).value and lib.tva_attn4_plan_splits(None) == -1


def _weigh(cache=None, **kw):
    a = evict.KeyWeightArgs()
    a.B, a.Hq, a.Hkv, a.D, a.max_rows, a.max_L, a.scale, a.ld = 2, 32, 8, 128, 4, 100, 0.1, 100
    a.cu_T = a.path = a.path_len = a.L = a.q = a.lse = a.weight = a.pos = a.first_pos = 4096
    a.cache = cache or _cache()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [(dict(B=-1), -1), (dict(Hq=12), -1), (dict(D=32), -2), (dict(max_rows=-1), -1), (dict(max_L=-1), -1),
                                     (dict(scale=-1.0), -1), (dict(ld=99), -1), (dict(cu_T=None), -1), (dict(path=None), -1), (dict(path_len=None), -1),
                                     (dict(L=None), -1), (dict(q=None), -1), (dict(q=4098), -1), (dict(lse=None), -1), (dict(weight=None), -1),
                                     (dict(first_pos=None), -1), (dict(B=65536), -2)])
def test_key_weights_refuse(lib, kw, code):
    assert lib.tva_key_weights(ctypes.byref(_weigh(**kw)), None) == code


def test_key_weights_of_nothing(lib):
    assert lib.tva_key_weights(None, None) == -1
    for kw in (dict(B=0), dict(max_rows=0), dict(max_L=0)):
        assert lib.tva_key_weights(ctypes.byref(_weigh(**kw)), None) == 0
    assert lib.tva_key_weights(ctypes.byref(_weigh(_cache(kind=cache4.ROWS_E4M3, k_scale=-1.0))), None) == -1
    assert lib.tva_key_weights(ctypes.byref(_weigh(_cache(kind=cache4.ROWS_E4M3, stride_tok=8))), None) == -1


def _select(**kw):
    a = evict.SelectArgs()
    a.n_layers, a.B, a.H, a.max_L, a.ld, a.ld_src = 1, 2, 8, 100, 100, 50
    a.L, a.keep, a.weight, a.src, a.L_out = 4096, 8192, 4096, 4096, 12288
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [(dict(B=-1), -1), (dict(H=0), -1), (dict(max_L=-1), -1), (dict(n_first=-1), -1), (dict(n_layers=-1), -1),
                                     (dict(max_L=262145, ld=262145), -2), (dict(ld=99), -1), (dict(ld_src=-1), -1), (dict(L=None), -1),
                                     (dict(keep=None), -1), (dict(weight=None), -1), (dict(src=None), -1), (dict(L_out=4096), -1), (dict(L_out=8192), -1),
                                     (dict(B=65536), -2), (dict(n_layers=65536), -2)])
def test_select_refuses(lib, kw, code):
    assert lib.tva_evict_select(ctypes.byref(_select(**kw)), None) == code
    assert lib.tva_evict_select(None, None) == -1 and lib.tva_evict_select(ctypes.byref(_select(B=0)), None) == 0


def _move(cache=None, **kw):
    a = evict.MoveArgs()
    a.n_layers, a.B, a.H, a.Hkv, a.D, a.max_keep, a.ld_src, a.ld = 1, 2, 8, 8, 128, 50, 50, 100
    a.n = a.src = a.weight = a.pos = 4096
    a.cache = cache or _cache()
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,code", [(dict(B=-1), -1), (dict(Hkv=0), -1), (dict(H=2), -1), (dict(H=0), -1), (dict(D=256), -2), (dict(max_keep=-1), -1),
                                     (dict(ld_src=49), -1), (dict(ld=49), -1), (dict(n=None), -1), (dict(src=None), -1), (dict(layer_stride_cache=-128), -1),
                                     (dict(layer_stride_cache=64), -1), (dict(n_layers=-1), -1), (dict(B=65536, H=1), -2), (dict(n_layers=65536), -2)])
def test_move_refuses(lib, kw, code):
    assert lib.tva_evict_move(ctypes.byref(_move(**kw)), None) == code
    assert lib.tva_evict_move(None, None) == -1 and lib.tva_evict_move(ctypes.byref(_move(max_keep=0)), None) == 0


def test_python_calls_refuse_shapes_that_do_not_fit(lib):
    import torch
    c = cache4.make_cache(k=torch.zeros(64, dtype=torch.uint8), cu_L=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        cache4.make_cache(k=torch.zeros(64, dtype=torch.uint8), cu_L=torch.zeros(2))
    rows, ints = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        cache4.make_rows_args(k_rows=rows, v_rows=rows, cu_T=ints[0, :2], L=ints[0], cache=c, max_rows=3, path=ints, path_len=ints[0])
    w = torch.zeros((1, 2, 8))
    with pytest.raises(ValueError):
        evict.make_key_weight_args(q=rows, lse=w, cache=c, cu_T=ints[0, :2], L=ints, weight=w, max_rows=4, max_L=8, scale=1.0, pos=w[..., :4])
    with pytest.raises(ValueError):
        evict.make_select_args(weight=w, L=ints, keep=ints, max_L=8, src=torch.zeros((2, 2, 8), dtype=torch.int32))
    with pytest.raises(ValueError):
        evict.make_move_args(src=torch.zeros((1, 2, 8), dtype=torch.int32), n=ints, cache=c, Hkv=2, D=64, max_keep=8, weight=torch.zeros((1, 1, 8)))
    with pytest.raises(TypeError):
        cache4.store_raw(evict.SelectArgs())
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="not contiguous"):
        evict.make_select_args(weight=torch.zeros((1, 2, 16))[..., :8], L=n, keep=n, max_L=8, src=torch.zeros((1, 2, 8), dtype=torch.int32))
    with pytest.raises(ValueError, match="int32"):
        evict.make_select_args(weight=w, L=n.long(), keep=n, max_L=8, src=torch.zeros((1, 2, 8), dtype=torch.int32))


def test_kernels_of_long_caches_keep_their_registers(lib):
    """No vector register goes to memory, and as many wavefronts fit as the kernels' workgroups per compute unit need."""
    from tests.test_kernel_resources import kernels
    most = {"four_bit_kernel": 256, "join_kernel": 128, "weigh_kernel": 170, "choose_kernel": 128, "shift_kernel": 64, "store_rows_kernel": 128,
            "load_rows_kernel": 64}
    seen = dict.fromkeys(most, 0)
    for name, k in kernels().items():
        for part, limit in most.items():
            if part in name:
                seen[part] += 1
                assert k[".vgpr_spill_count"] == 0 and k[".vgpr_count"] <= limit, (name, k[".vgpr_count"], k[".vgpr_spill_count"])
    assert all(seen.values()), seen
