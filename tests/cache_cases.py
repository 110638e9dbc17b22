"""Caches for the tests of include/tva_cache.h: values laid out the way a program keeps them, everything no sequence owns
filled with what would show."""
import numpy as np

from oracle import cache_oracle as orc


def trees(rng, sizes, depth=8):
    out = []
    for T in sizes:
        parent, deep = np.full(T, -1, np.int32), np.zeros(T, int)
        for i in range(1, T):
            p = int(rng.choice(np.nonzero(deep[:i] < depth)[0]))
            parent[i], deep[i] = p, deep[p] + 1
        out.append(parent)
    return out


def ancestor_sets(parent):
    seen = np.zeros((len(parent), len(parent)), bool)
    for i, p in enumerate(parent):
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def mask_words(seen, words):
    out = np.zeros((len(seen), words), np.uint64)
    for i, j in zip(*np.nonzero(seen)):
        out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out


def dev(x, dtype=None):
    import torch
    x = np.ascontiguousarray(x, dtype=dtype)
    if x.dtype == np.uint16:
        return torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)
    if x.dtype == np.uint64:
        x = x.view(np.int64)
    return torch.from_numpy(x).cuda()


def bits(t):
    """bf16 tensor -> uint16 patterns."""
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


class Layout:
    """Places for the positions of a batch: dense or paged, token-major or head-major.  room: positions per sequence."""

    def __init__(self, rng, room, Hkv, D, page=0, head_major=False):
        self.page, self.Hkv, self.D, B = page, Hkv, D, len(room)
        if page:
            n = [-(-int(r) // page) for r in room]
            self.table = np.full((B, max(1, max(n))), -1, np.int32)
            pool = rng.permutation(sum(n) + 3)
            at = 0
            for b, k in enumerate(n):
                self.table[b, :k] = pool[at:at + k]
                at += k
            self.rows = len(pool) * page * Hkv
            self.st = (page * Hkv, 1, page) if head_major else (page * Hkv, Hkv, 1)
            self.cu = None
        else:
            self.table, self.cu = None, np.concatenate([[0], np.cumsum(room)]).astype(np.int32)
            total = int(self.cu[-1]) + 2
            self.rows = total * Hkv
            self.st = (0, 1, total) if head_major else (0, Hkv, 1)
        self.d_cu, self.d_table = (None if x is None else dev(x) for x in (self.cu, self.table))

    def at(self, b, t):
        """Row numbers of positions t of sequence b, [len(t), Hkv]."""
        t = np.asarray(t)
        if self.page:
            base = self.table[b, t // self.page].astype(np.int64) * self.st[0] + t % self.page * self.st[1]
        else:
            base = (int(self.cu[b]) + t) * self.st[1]
        return base[:, None] + np.arange(self.Hkv) * self.st[2]

    def cache(self, **kw):
        from paper_2510_26577_amd import cache4
        return cache4.make_cache(cu_L=self.d_cu, page_table=self.d_table, page_size=self.page, strides=tuple(s * self.D for s in self.st), **kw)


class FourBit:
    """A cache of random 4-bit rows; rows of no sequence hold the largest values there are, and NaN scales."""

    def __init__(self, rng, lay, lengths, layers=1, spread=1.0):
        D = lay.D
        n = lay.rows * layers
        self.lay, self.lengths = lay, lengths
        self.k = rng.integers(0, 256, (n, D // 2)).astype(np.uint8)
        self.v = rng.integers(0, 256, (n, D // 2)).astype(np.uint8)
        self.ks = np.full((n, D // 32), 250, np.uint8)
        self.vs = np.full(n, 0x7FC0, np.uint16)  # NaN
        for layer in range(layers):
            for b, L in enumerate(lengths):
                r = lay.at(b, np.arange(L)) + layer * lay.rows
                self.ks[r] = rng.integers(125, 128, (*r.shape, D // 32)) + int(np.log2(spread))
                self.vs[r] = orc.to_bf16(np.ldexp(rng.integers(8, 16, r.shape) / 16.0, rng.integers(-2, 1, r.shape)))
        self.upload()

    def upload(self):
        self.d = dict(k=dev(self.k), v=dev(self.v), k_row_scale=dev(self.ks), v_row_scale=dev(self.vs))
        self.cache = self.lay.cache(**self.d)

    def download(self):
        return self.d["k"].cpu().numpy(), self.d["k_row_scale"].cpu().numpy(), self.d["v"].cpu().numpy(), bits(self.d["v_row_scale"])

    def values(self, b, t, layer=0):
        r = self.lay.at(b, t) + layer * self.lay.rows
        return orc.decode_k(self.k[r], self.ks[r]), orc.decode_v(self.v[r], self.vs[r])
