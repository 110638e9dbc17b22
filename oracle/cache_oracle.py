"""Independent CPU oracle of include/tva_cache.h: 4-bit rows, the attention over them, attention weights of keys, the choice
of slots.  Plain numpy in 64 bits, one sequence at a time; test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def bf16(x):
    """uint16 patterns -> float64 values."""
    return (np.asarray(x, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16(x):
    """float64 -> uint16 patterns, round to nearest even (finite values)."""
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def _scale(a, bits):
    """The smallest number of `bits` significant bits with a <= 6 s, within 2^-96 .. 2^124."""
    if a == 0.0:
        return 2.0 ** -96
    e = math.frexp(a)[1] - 3 - bits  # a step well below a / 6 for that many bits
    k = 1
    while True:  # steps of 2^e: k of at most `bits` bits
        if k >= 2 ** bits:
            k, e = 2 ** (bits - 1), e + 1
        if 6.0 * math.ldexp(k, e) >= a:
            break
        k += 1
    return min(max(math.ldexp(k, e), 2.0 ** -96), 2.0 ** 124)


def _code(x, s):
    if math.isnan(x):
        return 0
    a = min(abs(x) / s, 6.0) if math.isfinite(x) else 6.0
    near = min(range(8), key=lambda c: (abs(MAGNITUDES[c] - a), c & 1))
    return near | (8 if math.copysign(1.0, x) < 0 else 0)


def encode(x, group, bits):
    """One row (float64 [D]) -> codes [D], scales [D / group]."""
    codes, scales = [], []
    for g in range(0, len(x), group):
        part = [float(v) for v in x[g:g + group]]
        s = _scale(max([abs(v) for v in part if math.isfinite(v)], default=0.0), bits)
        codes += [_code(v, s) for v in part]
        scales.append(s)
    return np.array(codes, np.uint8), np.array(scales)


def encode_rows(k, v):
    """bf16 patterns [.., D] of K and V -> what the cache holds: k bytes [.., D/2], k scale bytes [.., D/32], v bytes, v scales
    (bf16 patterns [..])."""
    k, v = bf16(k), bf16(v)
    D, lead = k.shape[-1], k.shape[:-1]
    out = ([], [], [], [])
    for a, b in zip(k.reshape(-1, D), v.reshape(-1, D)):
        ck, sk = encode(a, 32, 1)
        cv, sv = encode(b, D, 4)
        out[0].append(ck[0::2] | ck[1::2] << 4)
        out[1].append([int(math.log2(s)) + 127 for s in sk])
        out[2].append(cv[0::2] | cv[1::2] << 4)
        out[3].append(to_bf16(sv)[0])
    return (np.array(out[0], np.uint8).reshape(*lead, D // 2), np.array(out[1], np.uint8).reshape(*lead, D // 32),
            np.array(out[2], np.uint8).reshape(*lead, D // 2), np.array(out[3], np.uint16).reshape(lead))


def decode(x):
    """Bytes [.., n] -> the codes' values [.., 2 n]."""
    x = np.asarray(x, np.uint8)
    c = np.stack([x & 15, x >> 4], -1).reshape(*x.shape[:-1], 2 * x.shape[-1])
    return np.array(MAGNITUDES)[c & 7] * np.where(c & 8, -1.0, 1.0)


def decode_k(x, scale):
    return decode(x) * np.repeat(2.0 ** (np.asarray(scale, np.float64) - 127), 32, -1)


def decode_v(x, scale):
    return decode(x) * bf16(scale)[..., None]


def attention(q, K, V, seen, scale):
    """q [n, Hq, D], K and V [keys, Hkv, D], seen [n, keys] -> out, lse, and per row sum p |V| (like out) and the largest
    scale * sum |q| |k| (like lse), which bound what roundings can do."""
    n, Hq, D = q.shape
    G = Hq // K.shape[1]
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    size, reach = np.zeros((n, Hq, D)), np.zeros((n, Hq))
    for i in range(n):
        if not seen[i].any():
            continue
        for h in range(Hq):
            k, v = K[seen[i], h // G], V[seen[i], h // G]
            x = scale * (k @ q[i, h])
            m = x.max()
            lse[i, h] = m + np.log(np.exp(x - m).sum())
            p = np.exp(x - lse[i, h])
            out[i, h], size[i, h] = p @ v, p @ np.abs(v)
            reach[i, h] = scale * (np.abs(k) @ np.abs(q[i, h])).max()
    return out, lse, size, reach


def key_weights(weight, q, lse, K, n, scale):
    """weight [Hkv, L] before; q [n, Hq, D], lse [n, Hq] of the newest n tokens; K [L, Hkv, D] -> weight after, and what bounds
    its error: the sum of the added weights times scale * sum |q| |k|."""
    Hkv, L = weight.shape
    G = q.shape[1] // Hkv
    w, off = weight.astype(np.float64).copy(), np.zeros_like(weight, np.float64)
    w[:, L - n:] = 0.0
    for i in range(n):
        end = L - n + i + 1
        for h in range(q.shape[1]):
            if lse[i, h] == -np.inf:
                continue
            p = np.exp(scale * (K[:end, h // G] @ q[i, h]) - lse[i, h])
            w[h // G, :end] += p
            off[h // G, :end] += p * (scale * (np.abs(K[:end, h // G]) @ np.abs(q[i, h])) + abs(lse[i, h]) + 1)
    return w, off


def select(weight, keep, n_first=0, newest=None, pos=None):
    """One row: weight [L] -> src [n]."""
    L = len(weight)
    n = max(0, min(int(keep), L))
    age = np.arange(L) if pos is None else pos

    def order(t):
        if t < n_first or (newest is not None and age[t] >= newest):
            return (0, 0.0, t)
        w = float(weight[t])
        return (2, 0.0, t) if math.isnan(w) else (1, -w, t)

    kept = set(sorted(range(L), key=order)[:n])
    src = np.arange(n)
    src[[t for t in range(n) if t not in kept]] = [t for t in range(n, L) if t in kept]
    return src.astype(np.int32)
