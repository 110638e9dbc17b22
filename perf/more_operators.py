"""Operators of new tokens on their way through a layer, as timed cases, each in its plain form and as a user calls the library.

  rotate   rotary positions of the heads of q and k (pairs half a head apart, or side by side; all of a head or its first
           part; frequencies stretched for long contexts), the norm of every head in the same pass where the model has one
  append   k (normed, rotated) and v to the end of every sequence's cache: 16-bit, 8-bit or 4-bit rows, dense or in pages;
           q rotated beside them
  attn     the attention of the new tokens, which the cache holds already: a chunk of a prompt (causal) or a draft tree
           (ancestors), over everything or over a window and the first few tokens

Sizes: batch 1 .. 64, trees of at most 72 nodes, chunks of at most 16384 tokens, caches of at most 32768, positions to half a million.
"""
import math

import numpy as np
import torch

own = False

HEADS = {"4/4/64": (4, 4, 64), "16/8/128": (16, 8, 128), "24/8/128": (24, 8, 128), "32/8/64": (32, 8, 64),
         "32/8/128": (32, 8, 128), "64/8/128": (64, 8, 128)}
DEV = "cuda"


def listed():
    return [
        # interactive use: a full draft tree's queries and keys, positions by depth (latency counts)
        dict(name="rotate_tree", kind="rotate", heads="32/8/128", B=1, T=60, tree=True, L=2048, dims=128, interleaved=False, scaling="none", norm=False),
        # chunks far into long contexts, pairs side by side in half of the head, frequencies stretched
        dict(name="rotate_long", kind="rotate", heads="64/8/128", B=4, T=2051, tree=False, L=300000, dims=64, interleaved=True, scaling="ramp", norm=False),
        # plain decoding of a batch, a model with norms of its heads
        dict(name="norm_tokens", kind="rotate", heads="32/8/128", B=64, T=1, tree=False, L=4000, dims=128, interleaved=False, scaling="none", norm=True),
        # a whole prompt through such a layer
        dict(name="norm_prompt", kind="rotate", heads="32/8/128", B=1, T=16384, tree=False, L=0, dims=128, interleaved=False, scaling="wavelength", norm=True),
        # the step of a batch in plain decoding: q, k and v of its tokens, an 8-bit cache in pages
        dict(name="append_tokens", kind="append", heads="32/8/128", B=64, T=1, tree=False, L=1000, dims=128, interleaved=False, scaling="none", norm=False,
             rows="e4m3", page=16, head_major=False),
        # prompts on their way into a cache of 4-bit rows, and read back
        dict(name="append_prompts", kind="append", heads="32/8/128", B=4, T=4099, tree=False, L=0, dims=128, interleaved=False, scaling="linear",
             norm=True, rows="e2m1", page=16, head_major=True),
        # the first prompt of one sequence
        dict(name="chunk_first", kind="attn", heads="32/8/128", B=1, T_lo=2048, T_hi=2048, tree=False, L_lo=0, L_hi=0, window=0, first=0, rows="bf16",
             page=16, head_major=False),
        # a chunk of a long prompt
        dict(name="chunk_long", kind="attn", heads="32/8/128", B=1, T_lo=2048, T_hi=2048, tree=False, L_lo=30000, L_hi=30000, window=0, first=0,
             rows="bf16", page=64, head_major=False),
        # requests of all lengths scheduled together, an 8-bit cache
        dict(name="chunk_ragged", kind="attn", heads="32/8/128", B=16, T_lo=1, T_hi=333, tree=False, L_lo=100, L_hi=8000, window=0, first=0,
             rows="e4m3", page=16, head_major=False),
        # plain decoding of a large batch, a layer that sees a window
        dict(name="window_tokens", kind="attn", heads="32/8/128", B=64, T_lo=1, T_hi=1, tree=False, L_lo=4096, L_hi=16384, window=1024, first=4,
             rows="bf16", page=16, head_major=False),
        # a draft tree in such a layer
        dict(name="window_tree", kind="attn", heads="32/8/128", B=1, T_lo=60, T_hi=60, tree=True, L_lo=8192, L_hi=8192, window=4096, first=4,
             rows="bf16", page=0, head_major=False),
        # a long prompt's chunk in such a layer
        dict(name="window_prompt", kind="attn", heads="32/8/128", B=1, T_lo=8192, T_hi=8192, tree=False, L_lo=8192, L_hi=8192, window=4096, first=4,
             rows="bf16", page=0, head_major=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "append", "append", "attn", "attn", "attn", "attn"])
    heads = rng.choice(["4/4/64", "16/8/128", "24/8/128", "32/8/64", "32/8/128", "32/8/128", "64/8/128"])
    Hq, Hkv, D = HEADS[heads]
    B = _log_int(rng, 1, 64)
    tree = rng.random() < 0.35
    if kind == "attn":
        most = 2048 * 32048 * 32 // Hq  # scores: the longest chunk's
        T = _log_int(rng, 1, 72 if tree else min(8192, 40000 // B, math.isqrt(most // B)))
        hi = min(32768, 400_000 // B, most // (B * T) - T)
        L = _log_int(rng, 1, max(1, hi)) - (0 if rng.random() < 0.8 else 1)
        window = rng.choice([0, _log_int(rng, 1, 8192)])
        return dict(kind=kind, heads=heads, B=B, T_lo=T if rng.random() < 0.4 else max(1, int(T * rng.random())), T_hi=T, tree=tree,
                    L_lo=L if rng.random() < 0.4 else int(L * rng.random()), L_hi=L, window=window, first=rng.choice([0, 1, 4, 70]) if window else 0,
                    rows=rng.choice(["bf16", "bf16", "e4m3"]), page=rng.choice([0, 16, 24, 64]), head_major=rng.random() < 0.4)
    T = _log_int(rng, 1, 72 if tree else 16384 // B)
    both = dict(kind=kind, heads=heads, B=B, T=T, tree=tree, dims=rng.choice([D, D, D // 2, 16, 48]), interleaved=rng.random() < 0.4,
                scaling=rng.choice(["none", "linear", "base", "wavelength", "ramp"]), norm=rng.random() < 0.4)
    if kind == "rotate":
        return dict(both, L=_log_int(rng, 1, 500_000) - 1)
    return dict(both, L=rng.randint(0, 300), rows=rng.choice(["bf16", "bf16", "e4m3", "e2m1"]), page=rng.choice([0, 16, 24, 64]),
                head_major=rng.random() < 0.4)


# ---- inputs ----
def _dev(x, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=dtype)).to(DEV)


def _normal(gen, shape):
    """Activations: N(0, 1) rounded once to bf16."""
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _spread(rng, lo, hi, B):
    return rng.permutation(np.linspace(hi, lo, B).round()).astype(np.int32)


def _masks(rng, sizes, words):
    """Ancestor sets of random trees of at most 9 levels, a root each: int64 [nodes, words]."""
    out = []
    for T in sizes:
        depth, rows = np.zeros(T, np.int64), []
        for i in range(T):
            p = int(rng.choice(np.nonzero(depth[:i] < 8)[0])) if i else -1
            depth[i] = depth[p] + 1 if i else 0
            rows.append((rows[p] if i else 0) | (1 << i))
        out += [[(r >> (64 * w)) & (2 ** 64 - 1) for w in range(words)] for r in rows]
    return np.array(out, np.uint64).reshape(-1, words).view(np.int64)


def _place(case, rng, room, Hkv):
    """Where positions lie: row number = page * strides[0] + slot * strides[1] + head * strides[2] (in rows of one head)."""
    B, ps = len(room), case["page"]
    if ps:
        n = [max(1, -(-int(l) // ps)) for l in room]
        pool = rng.permutation(int(math.ceil(1.25 * sum(n)))).astype(np.int32)
        table = np.zeros((B, max(n)), np.int32)
        at = 0
        for b, k in enumerate(n):
            table[b, :k] = pool[at:at + k]
            at += k
        st = (ps * Hkv, 1, ps) if case["head_major"] else (ps * Hkv, Hkv, 1)
        return dict(page_table=_dev(table), cu_L=None, page=ps, strides=st, rows=len(pool) * ps * Hkv)
    cu = np.concatenate([[0], np.cumsum(room)]).astype(np.int32)
    st = (0, 1, int(cu[-1])) if case["head_major"] else (0, Hkv, 1)
    return dict(page_table=None, cu_L=_dev(cu), page=0, strides=st, rows=max(1, int(cu[-1])) * Hkv)


def _row_numbers(place, pos, Hkv):
    """pos [B, n] -> [B, n, Hkv]."""
    sp, st, sh = place["strides"]
    if place["page"]:
        at = (pos // place["page"]).clamp(max=place["page_table"].shape[1] - 1).long()
        r = place["page_table"].gather(1, at).long() * sp + pos % place["page"] * st
    else:
        r = (place["cu_L"][:-1, None].long() + pos) * st
    return (r[..., None] + torch.arange(Hkv, device=pos.device) * sh).clamp(max=place["rows"] - 1)


def _frequencies(case):
    """Radians per position of every pair, and the factor of what is rotated: a model's constants."""
    r, base, factor, original = case["dims"], 10000.0, 8.0, 8192.0
    i = np.arange(r // 2)
    f, m = base ** (-2.0 * i / r), 1.0
    if case["scaling"] == "linear":
        f = f / factor
    elif case["scaling"] == "base":
        f = (base * factor ** (r / (r - 2.0))) ** (-2.0 * i / r)
    elif case["scaling"] == "wavelength":
        keep = np.clip((original * f / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = f * keep + f / factor * (1 - keep)
    elif case["scaling"] == "ramp":
        at = [r * math.log(original / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        keep = 1 - np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        f, m = f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0
    return f, m


def _own_cache(s, D, kind):
    from paper_2510_26577_amd import cache4
    p = s["place"]
    more = {}
    if kind == "e2m1":
        more = dict(k_row_scale=s["ks"], v_row_scale=s["vs"])
    elif kind == "e4m3":
        more = dict(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return cache4.make_cache(kind={"bf16": cache4.ROWS_BF16, "e4m3": cache4.ROWS_E4M3, "e2m1": cache4.ROWS_E2M1}[kind], k=s["k"], v=s["v"],
                             cu_L=p["cu_L"], page_table=p["page_table"], page_size=p["page"], strides=tuple(x * D for x in p["strides"]), **more)


def _prepare_new(case, rng, gen):
    """rotate and append: what the layer's projection gave, a token's heads of q, k and v side by side."""
    Hq, Hkv, D = HEADS[case["heads"]]
    B, T, append = case["B"], case["T"], case["kind"] == "append"
    sizes = rng.permutation([max(1, T - b * (T // 8) // B) for b in range(B)])
    cu_T = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n, L = int(cu_T[-1]), case["L"] + rng.integers(0, 64, B)
    f, m = _frequencies(case)
    s = dict(kind=case["kind"], D=D, Hq=Hq, Hkv=Hkv, dims=case["dims"], interleaved=case["interleaved"], magnitude=m, eps=1e-6, width=int(max(sizes)),
             cu_T=_dev(cu_T), L=_dev(L, np.int32), freq=_dev(f, np.float64), mask=None, q_norm=None, k_norm=None,
             x=_normal(gen, (n, Hq + 2 * Hkv, D)), q_out=torch.zeros((n, Hq, D), dtype=torch.bfloat16, device=DEV))
    if case["tree"]:
        s["mask"] = _dev(_masks(rng, sizes, 1 + (max(sizes) > 64)))
    if case["norm"]:
        s["q_norm"], s["k_norm"] = (1 + 0.2 * _normal(gen, (D,)).float()).to(torch.bfloat16), (1 + 0.2 * _normal(gen, (D,)).float()).to(torch.bfloat16)
    s["q"], s["k_new"], s["v_new"] = s["x"][:, :Hq], s["x"][:, Hq:Hq + Hkv], s["x"][:, Hq + Hkv:]
    if append:
        s["rows"], s["place"] = case["rows"], _place(case, rng, [case["L"] + 64 + int(max(sizes))] * B, Hkv)
        rows, wide = s["place"]["rows"], {"bf16": D, "e4m3": D, "e2m1": D // 2}[case["rows"]]
        kind = {"bf16": torch.bfloat16, "e4m3": torch.uint8, "e2m1": torch.uint8}[case["rows"]]
        s["k"], s["v"] = (torch.zeros((rows, wide), dtype=kind, device=DEV) for _ in range(2))
        s["k_scale"], s["v_scale"] = 0.0125, 0.01
        if case["rows"] == "e2m1":
            s["ks"], s["vs"] = torch.zeros((rows, D // 32), dtype=torch.uint8, device=DEV), torch.zeros(rows, dtype=torch.bfloat16, device=DEV)
            s["k_back"], s["v_back"] = (torch.zeros((n, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        s["k_out"] = torch.zeros((n, Hkv, D), dtype=torch.bfloat16, device=DEV)
    if own:  # a program with fixed buffers fills the argument block once
        from paper_2510_26577_amd import cache4, rotary
        both = dict(q=s["q"], k=s["k_new"], q_out=s["q_out"], cu_T=s["cu_T"], L=s["L"], anc_mask=s["mask"], freq=s["freq"], dims=s["dims"],
                    interleaved=s["interleaved"], magnitude=m, q_norm=s["q_norm"], k_norm=s["k_norm"], eps=s["eps"])
        if append:
            cache = _own_cache(s, D, case["rows"])
            s["args"] = rotary.make_append_args(v=s["v_new"], cache=cache, **both)
            if case["rows"] == "e2m1":
                s["load"] = cache4.make_rows_args(k_rows=s["k_back"], v_rows=s["v_back"], cu_T=s["cu_T"], L=s["L"], cache=cache, max_rows=s["width"])
        else:
            s["args"] = rotary.make_rotate_args(k_out=s["k_out"], **both)
    return s


def _prepare_attn(case, rng, gen):
    Hq, Hkv, D = HEADS[case["heads"]]
    B, L = case["B"], _spread(rng, case["L_lo"], case["L_hi"], case["B"])
    sizes = _spread(rng, case["T_lo"], case["T_hi"], B)
    cu_T = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n, max_T = int(cu_T[-1]), int(max(sizes))
    s = dict(kind="attn", rows=case["rows"], Hkv=Hkv, G=Hq // Hkv, D=D, max_T=max_T, max_L=int(L.max()), window=case["window"], first=case["first"],
             scale=1.0 / math.sqrt(D), place=_place(case, rng, L + sizes, Hkv), cu_T=_dev(cu_T), L=_dev(L), mask=None, q=_normal(gen, (n, Hq, D)),
             k_scale=1.0, v_scale=1.0)
    if case["tree"]:
        s["mask"] = _dev(_masks(rng, sizes, 1 + (max_T > 64)))
    s["k"], s["v"] = (_normal(gen, (s["place"]["rows"], D)) for _ in range(2))
    if case["rows"] == "e4m3":
        s["k_scale"], s["v_scale"] = 0.0125, 0.01
        s["k"], s["v"] = ((x.float() / c).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x, c in ((s["k"], 0.0125), (s["v"], 0.01)))
    if own:
        from paper_2510_26577_amd import chunk
        s["out"], s["lse"] = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=DEV), torch.empty((n, Hq), dtype=torch.float32, device=DEV)
        s["args"] = chunk.make_args(q=s["q"], cache=_own_cache(s, D, case["rows"]), cu_T=s["cu_T"], L=s["L"], Hkv=Hkv, max_T=max_T, max_L=s["max_L"],
                                    scale=s["scale"], window=s["window"], n_first=s["first"], anc_mask=s["mask"], out=s["out"], lse=s["lse"])
        s["ws"] = chunk.attn_workspace(s["args"], DEV)
    return s


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return (_prepare_attn if case["kind"] == "attn" else _prepare_new)(case, rng, gen)


# ---- the plain forms ----
def _bits(mask):
    """How many bits of each row are set, [nodes]."""
    j = torch.arange(64, device=mask.device)
    return ((mask[..., None] >> j) & 1).sum((-1, -2))


def _positions(s):
    n = s["x"].shape[0]
    r = torch.arange(n, device=s["L"].device, dtype=torch.int32)
    b = torch.searchsorted(s["cu_T"][1:].contiguous(), r, right=True)
    i = r - s["cu_T"][b]
    return b, i, s["L"][b] + (i if s["mask"] is None else _bits(s["mask"]) - 1)


def _rotated(s, x, weight, cos, sin):
    """x bf16 [n, H, D] -> fp32, normed and rotated."""
    x, r = x.float(), s["dims"]
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight.float()
    a, rest = x[..., :r], x[..., r:]
    u, v = (a[..., 0::2], a[..., 1::2]) if s["interleaved"] else (a[..., :r // 2], a[..., r // 2:])
    y = (u * cos - v * sin, v * cos + u * sin)
    a = torch.stack(y, -1).flatten(-2) if s["interleaved"] else torch.cat(y, -1)
    return torch.cat([a, rest], -1)


def _both_rotated(s, pos):
    angle = pos.double()[:, None, None] * s["freq"]
    cos, sin = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    return _rotated(s, s["q"], s["q_norm"], cos, sin).to(torch.bfloat16), _rotated(s, s["k_new"], s["k_norm"], cos, sin).to(torch.bfloat16)


def _plain_rotate(s):
    q, k = _both_rotated(s, _positions(s)[2])
    s["q_out"].copy_(q)
    s["k_out"].copy_(k)
    return s["q_out"], s["k_out"]


def _code(x, s):
    """E2M1 codes of x / s: half-way values go to the even code."""
    a = x.abs()
    c = (a > 0.25 * s).int() + (a >= 0.75 * s) + (a > 1.25 * s) + (a >= 1.75 * s) + (a > 2.5 * s) + (a >= 3.5 * s) + (a > 5.0 * s)
    return c + 8 * torch.signbit(x)


def _pack(c):
    return (c[..., 0::2] + 16 * c[..., 1::2]).to(torch.uint8)


def _round_k(x):
    """fp32 [.., D] -> bytes [.., D/2], scale bytes [.., D/32]: a power of two for 32 elements."""
    g = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1))
    e = torch.where(m == 0, -96, (e - 3 + (m > 0.75)).clamp(-96, 124))
    c = _code(g, torch.ldexp(torch.ones_like(m), e)[..., None])
    return _pack(c.flatten(-2)), (e + 127).to(torch.uint8)


def _round_v(x):
    """fp32 [.., D] -> bytes [.., D/2], scales bf16 [..] of four significant bits."""
    m, e = torch.frexp(x.abs().amax(-1))
    k = torch.where(m < 0.75, torch.ceil(m * 128 / 6) / 128, torch.ceil(m * 64 / 6) / 64)
    s = torch.ldexp(k, e).clamp(2.0 ** -96, 2.0 ** 124)
    return _pack(_code(x, s[..., None])), s.to(torch.bfloat16)


def _values(x):
    """Bytes -> the values of their codes, fp32, twice as long."""
    v = torch.tensor((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0), device=x.device)
    return torch.stack([v.repeat(16), v.repeat_interleave(16)], 1)[x.int()].flatten(-2)


def _eight(x, scale):
    return (x.float() / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    b, i, pos = _positions(s)
    q, k = _both_rotated(s, pos)
    s["q_out"].copy_(q)
    j = torch.arange(s["width"], device=b.device)
    at = _row_numbers(s["place"], s["L"][:, None].long() + j, s["Hkv"])[b, i]
    v = s["v_new"]
    if s["rows"] == "bf16":
        s["k"][at], s["v"][at] = k, v
    elif s["rows"] == "e4m3":
        s["k"][at], s["v"][at] = _eight(k, s["k_scale"]), _eight(v, s["v_scale"])
    else:
        s["k"][at], s["ks"][at] = _round_k(k.float())
        s["v"][at], s["vs"][at] = _round_v(v.float())
        scale = torch.ldexp(torch.ones((), device=at.device), s["ks"][at].int() - 127)
        s["k_back"][:] = (_values(s["k"][at]).unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2).to(torch.bfloat16)
        s["v_back"][:] = (_values(s["v"][at]) * s["vs"][at].float()[..., None]).to(torch.bfloat16)
    return _appended(s)


def _appended(s):
    if s["rows"] == "e2m1":
        return s["q_out"], s["k_back"], s["v_back"]
    if s["rows"] == "e4m3":
        return s["q_out"], s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn)
    return s["q_out"], s["k"], s["v"]


def _plain_attn(s):
    B, Hkv, G, max_T, max_K = s["L"].shape[0], s["Hkv"], s["G"], s["max_T"], s["max_L"] + s["max_T"]
    dev = s["L"].device
    t, i = torch.arange(max_K, device=dev), torch.arange(max_T, device=dev)
    at = _row_numbers(s["place"], t.expand(B, -1), Hkv)
    node = (s["cu_T"][:-1, None].long() + i).clamp(max=s["q"].shape[0] - 1)  # [B, max_T], those past a chunk's end are left out below
    new = t - s["L"][:, None]  # [B, max_K]: which new token a slot holds, below 0 for cached ones
    inside = new < (s["cu_T"][1:] - s["cu_T"][:-1])[:, None]
    if s["mask"] is None:
        pos = s["L"][:, None] + i
        key_pos = t.expand(B, -1)
        seen = new[:, None] <= i[:, None]
    else:
        depth = (_bits(s["mask"])[node] - 1)
        pos = s["L"][:, None] + depth
        j = new.clamp(0, max_T - 1)
        key_pos = torch.where(new < 0, t, s["L"][:, None] + depth.gather(1, j))
        words = s["mask"][node].gather(2, (j // 64)[:, None].expand(-1, max_T, -1))
        seen = (new < 0)[:, None] | (((words >> (j % 64)[:, None]) & 1) != 0)
    seen = seen & inside[:, None]
    if s["window"]:
        seen = seen & ((key_pos[:, None] > pos[..., None] - s["window"]) | (key_pos < s["first"])[:, None])
    q = s["q"][node].float().unflatten(2, (Hkv, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B, Hkv, max_T * G, D]
    K, V = s["k"][at], s["v"][at]
    if s["rows"] == "e4m3":
        K, V = K.view(torch.float8_e4m3fn), V.view(torch.float8_e4m3fn)
    x = torch.matmul(q, (K.float() * s["k_scale"]).permute(0, 2, 3, 1).contiguous())
    x *= s["scale"]
    x.masked_fill_(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x -= torch.where(top == -math.inf, 0.0, top)
    x.exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, (V.float() * s["v_scale"]).permute(0, 2, 1, 3).contiguous()) / torch.where(total == 0, 1.0, total)
    ragged = lambda y: y.unflatten(2, (max_T, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # noqa: E731  [B, max_T, Hq, ..]
    r = torch.arange(s["q"].shape[0], device=dev, dtype=torch.int32)
    b = torch.searchsorted(s["cu_T"][1:].contiguous(), r, right=True)
    n = r - s["cu_T"][b]
    return ragged(out)[b, n].to(torch.bfloat16), ragged(top + torch.log(total))[b, n][..., 0]


def run(state):
    s = state
    if not own:
        return {"rotate": _plain_rotate, "append": _plain_append, "attn": _plain_attn}[s["kind"]](s)
    from paper_2510_26577_amd import cache4, chunk, rotary
    if s["kind"] == "rotate":
        rotary.rotate_raw(s["args"])
        return s["q_out"], s["k_out"]
    if s["kind"] == "append":
        rotary.append_raw(s["args"])
        if s["rows"] == "e2m1":
            cache4.load_raw(s["load"])
        return _appended(s)
    chunk.attn_raw(s["args"])
    return s["out"], s["lse"]


# ---- the definitions in 64 bits, sequence by sequence ----
def _exact_heads(s, x, weight, pos):
    x = x.double()
    if weight is not None:
        x = x * torch.rsqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / s["D"] + s["eps"]) * weight.double()
    r = s["dims"]
    first, second = (slice(0, r, 2), slice(1, r, 2)) if s["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(s["freq"], s["magnitude"]), s["freq"] * pos[:, None, None])
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_positions(s):
    out, at = [], 0
    for b, L in enumerate(s["L"].tolist()):
        n = int(s["cu_T"][b + 1]) - at
        if s["mask"] is None:
            out += [float(L + i) for i in range(n)]
        else:
            out += [float(L - 1 + sum(bin(w & (2 ** 64 - 1)).count("1") for w in words)) for words in s["mask"][at:at + n].tolist()]
        at += n
    return torch.tensor(out, dtype=torch.float64, device=DEV)


def _exact_rotate(s):
    pos = _exact_positions(s)
    return _exact_heads(s, s["q"], s["q_norm"], pos), _exact_heads(s, s["k_new"], s["k_norm"], pos)


def _slots(s, b, lo, hi):
    """Row numbers of sequence b's positions lo .. hi-1, [n, Hkv]."""
    p = s["place"]
    t = torch.arange(lo, hi, device=DEV)
    if p["page"]:
        base = p["page_table"][b].long()[t // p["page"]] * p["strides"][0] + t % p["page"] * p["strides"][1]
    else:
        base = (int(p["cu_L"][b]) + t) * p["strides"][1]
    return base[:, None] + torch.arange(s["Hkv"], device=DEV) * p["strides"][2]


def _exact_append(s):
    """(8-bit rows: before they are rounded.  Which of its few values a 4-bit element takes depends on which side of a border it falls: no value.)"""
    q, k = _exact_rotate(s)
    if s["rows"] == "e2m1":
        return q, None, None
    eight = s["rows"] == "e4m3"
    kc, vc = torch.zeros_like(s["k"], dtype=torch.float64), torch.zeros_like(s["v"], dtype=torch.float64)
    cu = s["cu_T"].tolist()
    for b, L in enumerate(s["L"].tolist()):
        at = _slots(s, b, L, L + cu[b + 1] - cu[b])
        kc[at], vc[at] = k[cu[b]:cu[b + 1]], s["v_new"][cu[b]:cu[b + 1]].double()
    if eight:
        kc, vc = (kc / s["k_scale"]).clamp(-448, 448), (vc / s["v_scale"]).clamp(-448, 448)
    return q, kc, vc


def _exact_attn(s):
    n, Hq = s["q"].shape[:2]
    out, lse = torch.empty((n, Hq, s["D"]), dtype=torch.float64, device=DEV), torch.empty((n, Hq), dtype=torch.float64, device=DEV)
    cu, G = s["cu_T"].tolist(), s["G"]
    for b, L in enumerate(s["L"].tolist()):
        lo, T = cu[b], cu[b + 1] - cu[b]
        at = _slots(s, b, 0, L + T)
        key = torch.arange(L + T, device=DEV)
        ok = torch.ones((T, L + T), dtype=torch.bool, device=DEV)
        if s["mask"] is None:
            ok[:, L:] = torch.tril(ok[:, L:])
            pos = key[L:]
        else:
            rows = [sum((w & (2 ** 64 - 1)) << (64 * k) for k, w in enumerate(words)) for words in s["mask"][lo:lo + T].tolist()]
            ok[:, L:] = torch.tensor([[(r >> j) & 1 == 1 for j in range(T)] for r in rows], device=DEV)
            pos = L - 1 + ok[:, L:].sum(1)
            key = torch.cat([key[:L], pos])
        if s["window"]:
            ok &= (pos[:, None] - key < s["window"]) | (key < s["first"])
        for g in range(s["Hkv"]):
            K, V = s["k"][at[:, g]], s["v"][at[:, g]]
            if s["rows"] == "e4m3":
                K, V = K.view(torch.float8_e4m3fn), V.view(torch.float8_e4m3fn)
            K, V = K.double() * s["k_scale"], V.double() * s["v_scale"]
            for h in range(g * G, (g + 1) * G):
                x = torch.where(ok, (s["q"][lo:lo + T, h].double() @ K.T) * s["scale"], -math.inf)
                z = torch.logsumexp(x, 1)
                out[lo:lo + T, h] = torch.exp(x - z[:, None]) @ V
                lse[lo:lo + T, h] = z
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "attn": _exact_attn}[case["kind"]](s)


# ---- what a pass cannot do without ----
def work(case):
    Hq, Hkv, D = HEADS[case["heads"]]
    B = case["B"]
    if case["kind"] != "attn":
        n = B * case["T"] if case["T"] < 8 else sum(max(1, case["T"] - b * (case["T"] // 8) // B) for b in range(B))
        rows = {"bf16": 4 * D, "e4m3": 2 * D, "e2m1": D + D // 32 + 2}[case["rows"]] * Hkv if case["kind"] == "append" else 0
        back = (rows + 4 * D * Hkv) if case["kind"] == "append" and case["rows"] == "e2m1" else 0
        heads = 2 * (Hq + Hkv) * 2 * D if case["kind"] == "rotate" else 2 * Hq * 2 * D + 2 * Hkv * 2 * D + rows + back
        return {"bytes": n * heads, "flops": n * (Hq + Hkv) * (3 * case["dims"] + (4 * D if case["norm"] else 0))}
    T, L = (np.linspace(case[x + "_hi"], case[x + "_lo"], B).round() for x in ("T", "L"))
    T, L = T.astype(np.int64), np.full(B, L.mean())  # (which lengths meet is drawn)
    W, one = case["window"] or 1 << 40, 2 if case["rows"] == "bf16" else 1
    keys = pairs = 0.0
    for n, l in zip(T, L):
        new = np.minimum(np.arange(n), 4) if case["tree"] else np.arange(n)  # about: a node's ancestors
        there = l + new + 1
        pairs += float((np.minimum(there, W) + np.clip(there - W, 0, case["first"])).sum())
        keys += float(min(l + n, W + n - 1 + np.clip(l + 1 - W, 0, case["first"])))
    return {"bytes": keys * Hkv * 2 * D * one + float(T.sum()) * Hq * (4 * D + 4), "flops": 4.0 * D * Hq * pairs}
