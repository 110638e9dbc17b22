"""The oracle of include/tva_layer.h against values worked out by hand, and the library's frequencies (a host function) against it (CPU)."""
import ctypes
import math

import numpy as np
import pytest

from oracle import fp8_oracle, layer_oracle as orc
from paper_2510_26577_amd import binding, rotary


def test_heads_turn_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]]])
    freq = np.array([math.pi / 2, math.pi])
    y, _ = orc.heads(x, [1], freq, 4)                       # pairs (0, 2) by a quarter, (1, 3) by a half
    assert np.allclose(y, [[[-3.0, -2.0, 1.0, -4.0, 5.0, 6.0]]], atol=1e-15)
    y, _ = orc.heads(x, [1], freq, 4, interleaved=True, magnitude=2.0)  # pairs (0, 1), (2, 3)
    assert np.allclose(y, [[[-4.0, 2.0, -6.0, -8.0, 5.0, 6.0]]], atol=1e-14)
    y, _ = orc.heads(x, [-1], freq, 4)                      # the other way round
    assert np.allclose(y, [[[3.0, -2.0, -1.0, -4.0, 5.0, 6.0]]], atol=1e-15)


def test_heads_are_normed_by_hand():
    y, _ = orc.heads([[[3.0, 4.0]]], [7], [0.0], 0, norm=np.array([1.0, 2.0]))
    assert np.allclose(y, [[[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]]])
    y, _ = orc.heads([[[0.0, 0.0]]], [7], [0.0], 0, norm=np.ones(2), eps=1e-6)
    assert not y.any()


def test_eight_bit_rows_by_hand():
    table = fp8_oracle.e4m3_decode_table()
    got = table[orc.eight_bit(np.array([1.0, 17.0, 19.0, 1e9, -np.inf, 500.0, 2.0 ** -10, 1.5 * 2.0 ** -9]), 1.0)]
    assert got.tolist() == [1.0, 16.0, 20.0, 448.0, -448.0, 448.0, 0.0, 2.0 ** -8]  # ties go to the even code
    assert orc.eight_bit(np.array([math.nan, -0.0]), 1.0).tolist() == [0, 128]
    assert table[orc.eight_bit(np.array([3.0]), 2.0)].tolist() == [1.5]


def test_windows_by_hand():
    ok, pos = orc.seen(4, 3)
    assert ok.astype(int).tolist() == [[1, 1, 1, 1, 1, 0, 0], [1, 1, 1, 1, 1, 1, 0], [1] * 7] and pos.tolist() == [4, 5, 6]
    ok, _ = orc.seen(4, 3, window=2, n_first=1)
    assert ok.astype(int).tolist() == [[1, 0, 0, 1, 1, 0, 0], [1, 0, 0, 0, 1, 1, 0], [1, 0, 0, 0, 0, 1, 1]]
    ok, _ = orc.seen(2, 2, window=1)
    assert ok.astype(int).tolist() == [[0, 0, 1, 0], [0, 0, 0, 1]]
    sets = np.array([[1, 0, 0, 0], [1, 1, 0, 0], [1, 0, 1, 0], [1, 1, 0, 1]], bool)  # depths 0, 1, 1, 2
    ok, pos = orc.seen(3, 4, window=2, n_first=1, sets=sets)
    assert pos.tolist() == [3, 4, 4, 5]
    assert ok.astype(int).tolist() == [[1, 0, 1, 1, 0, 0, 0], [1, 0, 0, 1, 1, 0, 0], [1, 0, 0, 1, 0, 1, 0], [1, 0, 0, 0, 1, 0, 1]]


def test_attention_by_hand():
    q = np.array([[[1.0]], [[0.0]], [[1.0]]])
    K, V = np.array([[[0.0]], [[math.log(3.0)]]]), np.array([[[1.0]], [[5.0]]])
    out, lse, _, _ = orc.attention(q, K, V, np.array([[1, 1], [1, 1], [0, 0]], bool), 1.0)
    assert np.allclose(out[:, 0, 0], [4.0, 3.0, 0.0]) and np.allclose(lse[:2, 0], [math.log(4.0), math.log(2.0)]) and lse[2, 0] == -np.inf
    V[1] = np.nan
    out, _, _, _ = orc.attention(q, K, V, np.array([[1, 1], [1, 0], [0, 0]], bool), 1.0)
    assert math.isnan(out[0, 0, 0]) and out[1, 0, 0] == 1.0


KINDS = {"plain": rotary.PLAIN, "linear": rotary.LINEAR, "base": rotary.BASE, "wavelength": rotary.WAVELENGTH, "ramp": rotary.RAMP}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("dims,base,factor,original", [(128, 10000.0, 8.0, 8192.0), (64, 500000.0, 32.0, 4096.0), (16, 10000.0, 1.0, 2048.0), (48, 1e6, 2.5, 100.0), (4, 10.0, 4.0, 64.0)])
def test_the_librarys_frequencies(kind, dims, base, factor, original):
    low, high = (1.0, 4.0) if kind == "wavelength" else (1.0, 32.0)
    got, m = rotary.frequencies(dims, base, scaling=KINDS[kind], factor=factor, original=original, low=low)
    want, wm = orc.frequencies(kind, dims, base, factor, original, low, high)
    assert np.allclose(got, want, rtol=1e-13, atol=0) and abs(m - wm) <= 1e-15 * wm


def test_scaled_frequencies_lie_between_the_plain_ones_and_those_divided():
    plain, _ = rotary.frequencies(128)
    assert plain[0] == 1.0
    for kind in ("linear", "base", "wavelength", "ramp"):
        f, _ = rotary.frequencies(128, scaling=KINDS[kind], factor=8.0, original=8192.0)
        assert (f <= plain * (1 + 1e-15)).all() and (f >= plain / 8 * (1 - 1e-14)).all()
        assert abs(f[-1] / plain[-1] - 0.125) < 1e-12 and (f[0] == 1.0 or kind == "linear")


@pytest.mark.parametrize("bad", [dict(dims=6, base=1.0), dict(dims=2), dict(dims=5), dict(dims=0), dict(dims=8, base=math.nan), dict(dims=8, scaling=5), dict(dims=8, scaling=-1),
                                 dict(dims=8, scaling=1, factor=0.5), dict(dims=8, scaling=2, factor=math.inf), dict(dims=8, scaling=3, factor=2.0),
                                 dict(dims=8, scaling=4, factor=2.0, original=64.0, low=4.0, high=4.0), dict(dims=8, scaling=3, factor=2.0, original=64.0, low=0.0)])
def test_frequencies_that_are_none_are_refused(bad):
    with pytest.raises((ValueError, binding.TvaError)):
        rotary.frequencies(**bad)


def test_frequencies_without_a_place_are_refused():
    lib = rotary._lib()
    assert lib.tva_rotary_frequencies(0, 8, 10000.0, 1.0, 0.0, 0.0, 0.0, None, None) == -1
    freq = (ctypes.c_double * 4)()
    assert lib.tva_rotary_frequencies(0, 8, 10000.0, 1.0, 0.0, 0.0, 0.0, freq, None) == 0 and freq[0] == 1.0
