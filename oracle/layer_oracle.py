"""Independent CPU oracle of include/tva_layer.h: rotary positions, norms of heads, rows of an 8-bit cache, attention of new tokens with and
without a window.  Plain numpy in 64 bits, one sequence at a time; test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

from . import fp8_oracle


def frequencies(kind, dims, base, factor=1.0, original=0.0, low=0.0, high=0.0):
    """kind: the word that include/tva_layer.h names -> ([dims/2], magnitude), pair by pair from its definition."""
    if kind == "base":
        base = base * factor ** (dims / (dims - 2))
    out = []
    for j in range(dims // 2):
        f = 1.0 / base ** (2 * j / dims)
        if kind == "linear":
            f = f / factor
        elif kind == "wavelength":
            turns = original * f / (2 * math.pi)
            mix = 0.0 if turns <= low else 1.0 if turns >= high else (turns - low) / (high - low)
            f = mix * f + (1 - mix) * f / factor
        elif kind == "ramp":
            pair = lambda n: dims * math.log(original / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
            a, b = max(0, math.floor(pair(high))), min(dims - 1, math.ceil(pair(low)))
            mix = 1.0 if j <= a else 0.0 if j >= b else 1 - (j - a) / (b - a)
            f = mix * f + (1 - mix) * f / factor
        out.append(f)
    return np.array(out), 0.1 * math.log(factor) + 1.0 if kind == "ramp" else 1.0


def heads(x, pos, freq, dims, interleaved=False, magnitude=1.0, norm=None, eps=0.0):
    """x [n, H, D] (64 bits), pos [n] -> the normed and turned heads, and per element what roundings of 32 bits act on: the sizes of
    the two terms it is the sum of."""
    x = np.asarray(x, np.float64)
    if norm is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * norm
    y, size = x.copy(), np.abs(x)
    for j in range(dims // 2):
        u, v = (2 * j, 2 * j + 1) if interleaved else (j, j + dims // 2)
        for i, p in enumerate(np.asarray(pos).tolist()):
            turns = math.fmod(float(p) * float(freq[j]), 2 * math.pi)
            c, s = magnitude * math.cos(turns), magnitude * math.sin(turns)
            y[i, :, u] = x[i, :, u] * c - x[i, :, v] * s
            y[i, :, v] = x[i, :, v] * c + x[i, :, u] * s
            size[i, :, u] = size[i, :, v] = abs(magnitude) * (np.abs(x[i, :, u]) + np.abs(x[i, :, v]))
    return y, size


def eight_bit(x, scale):
    """Values (bf16 as float64) -> E4M3 codes of the fp32 quotient."""
    table = fp8_oracle.e4m3_decode_table()
    codes = np.array([c for c in range(256) if not math.isnan(table[c])])
    with np.errstate(over="ignore"):
        z = (np.asarray(x, np.float32) / np.float32(scale)).astype(np.float64)
    out = np.zeros(z.shape, np.uint8)
    for i in np.ndindex(z.shape):
        if math.isnan(z[i]):
            continue
        a = min(max(z[i], -448.0), 448.0)
        sign = 128 if math.copysign(1.0, a) < 0 else 0
        same = codes[(codes & 128) == sign]
        off = np.abs(table[same] - a)
        near = same[off == off.min()]
        out[i] = near[0] if len(near) == 1 else [c for c in near if c % 2 == 0][0]
    return out


def seen(L, T, window=0, n_first=0, sets=None, end=None):
    """Which of the L + T key slots each of T new tokens sees, [T, L + T]; sets [T, T]: a tree's.  end: slots that have a place."""
    ok = np.ones((T, L + T), bool)
    ok[:, L:] = np.tril(np.ones((T, T), bool)) if sets is None else sets
    pos = L + np.arange(T) if sets is None else L + np.asarray(sets).sum(1) - 1
    key = np.concatenate([np.arange(L), pos])
    if window:
        ok &= (key > pos[:, None] - window) | (key < n_first)
    if end is not None:
        ok[:, end:] = False
    return ok, pos


def attention(q, K, V, ok, scale):
    """q [n, Hq, D], K and V [keys, Hkv, D], ok [n, keys] -> out, lse, and what bounds roundings: per element the sum of p |V|, per row
    the largest scale * sum |q| |k|."""
    n, Hq, D = q.shape
    G = Hq // K.shape[1]
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    size, reach = np.zeros((n, Hq, D)), np.zeros((n, Hq))
    some = ok.any(1)
    if not some.any():
        return out, lse, size, reach
    for h in range(Hq):
        k, v = K[:, h // G], V[:, h // G]
        fine = np.where(np.isfinite(v), v, 0.0)
        x = np.where(ok, scale * (q[:, h] @ k.T), -np.inf)[some]
        m = x.max(1, keepdims=True)
        p = np.exp(x - m)
        total = p.sum(1, keepdims=True)
        p = p / total
        lse[some, h] = (m + np.log(total))[:, 0]
        o = p @ fine
        for j in np.nonzero(~np.isfinite(v).all(1))[0]:
            o[ok[some, j]] += np.where(np.isfinite(v[j]), 0.0, v[j])
        out[some, h], size[some, h] = o, p @ np.abs(fine)
        reach[some, h] = np.where(ok[some], scale * (np.abs(q[some, h]) @ np.abs(np.where(np.isfinite(k), k, 0.0)).T), 0.0).max(1)
    return out, lse, size, reach
