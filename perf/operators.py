"""Operators of long caches, as timed cases, each in its plain form and as a user calls the library.

  attn     the verification attention over a cache of 4-bit rows (single tokens and draft trees, dense and paged)
  store    bf16 rows rounded to 4-bit rows of the cache, and read back: an accepted path in all layers, or a prompt
  weights  the attention weight every cached key has received, brought up to date with a step's accepted tokens
  select   which slots of each head stay, by weight, age and place
  move     the kept rows moved into the gaps, all layers of a model

A 4-bit row holds E2M1 codes (magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6), K with a power of two per 32 elements, V with one
scale of four significant bits per row.  Sizes: batch 1 .. 64, trees of at most 72 nodes, caches of 1 .. 32768 tokens.
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
        # interactive use, plain decoding: one token of one sequence, one layer (latency counts)
        dict(name="token_1", kind="attn", heads="32/8/128", B=1, L_lo=1024, L_hi=1024, T=1, page=0, head_major=False),
        # interactive use: one sequence, a full draft tree
        dict(name="tree_1", kind="attn", heads="32/8/128", B=1, L_lo=2048, L_hi=2048, T=60, page=0, head_major=False),
        # throughput serving with long contexts: the largest batch, small trees, a pool that keeps a head's keys together
        dict(name="batch_64", kind="attn", heads="32/8/128", B=64, L_lo=4096, L_hi=16384, T=8, page=64, head_major=True),
        # long contexts of unequal length in a pool of short pages, large trees
        dict(name="long_paged", kind="attn", heads="32/8/128", B=4, L_lo=16384, L_hi=32768, T=48, page=16, head_major=False),
        # the end of a step: the accepted nodes of a large batch, all layers of a model in one call
        dict(name="commit_64", kind="store", heads="32/8/128", B=64, T=8, path=True, L=257, layers=32, page=0, head_major=False),
        # prompts on their way into the cache, one layer
        dict(name="prompts", kind="store", heads="32/8/128", B=4, T=4099, path=False, L=0, layers=1, page=16, head_major=False),
        # one sequence's accepted tokens weigh a 16-bit cache
        dict(name="weigh_1", kind="weights", heads="32/8/128", B=1, L_lo=2048, L_hi=2048, T=60, n=4, rows="bf16", page=0),
        # long contexts in 4 bits
        dict(name="weigh_long", kind="weights", heads="32/8/128", B=16, L_lo=16384, L_hi=32768, T=16, n=5, rows="e2m1", page=16),
        # one sequence over its budget, all heads of all layers
        dict(name="select_1", kind="select", layers=32, B=1, H=8, L_lo=2304, L_hi=2304, keep=2048, first=4, recent=256, aged=False),
        # long contexts cut to half, after earlier evictions (slots are not in order of age)
        dict(name="select_long", kind="select", layers=16, B=4, H=8, L_lo=16384, L_hi=32768, keep=12000, first=4, recent=1000, aged=True),
        # the moves that follow such choices
        dict(name="move_1", kind="move", heads="32/8/128", layers=32, B=1, L=2304, keep=2048, rows="bf16"),
        dict(name="move_long", kind="move", heads="32/8/128", layers=8, B=4, L=32768, keep=16384, rows="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "store", "weights", "weights", "select", "move"])
    heads = rng.choice(["4/4/64", "16/8/128", "24/8/128", "32/8/64", "32/8/128", "32/8/128", "64/8/128"])
    Hq, Hkv, D = HEADS[heads]
    B = _log_int(rng, 1, 64)
    if kind == "attn":
        T = _log_int(rng, 1, 72)
        hi = _log_int(rng, 1, max(1, min(32768, 600_000 // B, int(4_500_000 * 32 / Hq) // (B * T))))
        return dict(kind=kind, heads=heads, B=B, L_lo=hi if rng.random() < 0.3 else max(1, int(hi * rng.uniform(0.25, 1.0))), L_hi=hi, T=T,
                    page=rng.choice([0, 0, 16, 32, 64]), head_major=rng.random() < 0.5)
    if kind == "store":
        path = rng.random() < 0.5
        T = _log_int(rng, 1, 72) if path else _log_int(rng, 1, 16000 // B)
        return dict(kind=kind, heads=heads, B=B, T=T, path=path, L=rng.randint(0, 300), layers=rng.randint(1, 32) if path else 1,
                    page=rng.choice([0, 16, 32]), head_major=rng.random() < 0.5)
    if kind == "weights":
        T = _log_int(rng, 4, 72)
        n = rng.randint(1, min(T, 12))
        hi = _log_int(rng, n, max(n + 1, min(32768, 390_000 // B)))
        return dict(kind=kind, heads=heads, B=B, L_lo=max(n, int(hi * rng.uniform(0.3, 1.0))), L_hi=hi, T=T, n=n,
                    rows=rng.choice(["bf16", "e4m3", "e2m1"]) if D == 128 else rng.choice(["bf16", "e2m1"]), page=rng.choice([0, 16, 64]))
    layers = rng.randint(1, 16)
    L = _log_int(rng, 32, max(64, min(32768, (1_500_000 if kind == "select" else 110_000) // (B * layers))))
    keep = max(1, int(L * rng.uniform(0.3, 1.0)))
    if kind == "select":
        return dict(kind=kind, layers=layers, B=B, H=rng.choice([1, 4, 8]), L_lo=max(1, L // 2), L_hi=L, keep=keep, first=rng.randint(0, 4),
                    recent=rng.randint(0, keep), aged=rng.random() < 0.5)
    return dict(kind=kind, heads=heads, layers=layers, B=B, L=L, keep=keep, rows=rng.choice(["bf16", "e4m3"]) if D == 128 else "bf16")


# ---- 4-bit rows, elementary ----
_MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _code(x, s):
    """Codes of x / s: half-way values go to the even code."""
    a = x.abs()
    c = (a > 0.25 * s).int() + (a >= 0.75 * s) + (a > 1.25 * s) + (a >= 1.75 * s) + (a > 2.5 * s) + (a >= 3.5 * s) + (a > 5.0 * s)
    return c + 8 * torch.signbit(x)


def _pack(c):
    return (c[..., 0::2] + 16 * c[..., 1::2]).to(torch.uint8)


def _round_k(x):
    """fp32 [.., D] -> bytes [.., D/2], scale bytes [.., D/32]."""
    g = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(g.abs().amax(-1))
    e = torch.where(m == 0, -96, (e - 3 + (m > 0.75)).clamp(-96, 124))
    c = _code(g, torch.ldexp(torch.ones_like(m), e)[..., None])
    return _pack(c.flatten(-2)), (e + 127).to(torch.uint8)


def _round_v(x):
    """fp32 [.., D] -> bytes [.., D/2], scales bf16 [..]."""
    m, e = torch.frexp(x.abs().amax(-1))
    k = torch.where(m < 0.75, torch.ceil(m * 128 / 6) / 128, torch.ceil(m * 64 / 6) / 64)
    s = torch.ldexp(k, e).clamp(2.0 ** -96, 2.0 ** 124)
    return _pack(_code(x, s[..., None])), s.to(torch.bfloat16)


def _values(x):
    """Bytes -> the values of their codes, fp32, twice as long."""
    v = torch.tensor(_MAGNITUDES + tuple(-m for m in _MAGNITUDES), device=x.device)
    pairs = torch.stack([v.repeat(16), v.repeat_interleave(16)], 1)
    return pairs[x.int()].flatten(-2)


def _k_values(x, scale):
    v = _values(x).unflatten(-1, (-1, 32))
    return (v * torch.ldexp(torch.ones_like(scale, dtype=torch.float32), scale.int() - 127)[..., None]).flatten(-2)


def _v_values(x, scale):
    return _values(x) * scale.float()[..., None]


# ---- inputs ----
def _dev(x, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=dtype)).to(DEV)


def _normal(gen, shape):
    """Activations: N(0, 1) rounded once to bf16."""
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _lengths(case, rng):
    return rng.permutation(np.linspace(case["L_hi"], case["L_lo"], case["B"]).round()).astype(np.int32)


def _place(case, rng, room, Hkv):
    """Where positions lie: row number = page * strides[0] + slot * strides[1] + head * strides[2] (in rows of one head)."""
    B, ps = len(room), case["page"]
    if ps:
        n = [max(1, -(-int(l) // ps)) for l in room]
        pool = rng.permutation(int(math.ceil(1.25 * sum(n)))).astype(np.int32)
        table = np.full((B, max(n)), -1, np.int32)
        at = 0
        for b, k in enumerate(n):
            table[b, :k] = pool[at:at + k]
            at += k
        rows = len(pool) * ps
        st = (ps * Hkv, 1, ps) if case.get("head_major") else (ps * Hkv, Hkv, 1)
        return dict(page_table=_dev(table), cu_L=None, page=ps, strides=st, rows=rows * Hkv)
    cu = np.concatenate([[0], np.cumsum(room)]).astype(np.int32)
    st = (0, 1, int(cu[-1])) if case.get("head_major") else (0, Hkv, 1)
    return dict(page_table=None, cu_L=_dev(cu), page=0, strides=st, rows=max(1, int(cu[-1])) * Hkv)


def _row_numbers(place, pos, Hkv):
    """pos [B, n] -> [B, n, Hkv]."""
    sp, st, sh = place["strides"]
    if place["page"]:
        at = (pos // place["page"]).clamp(max=place["page_table"].shape[1] - 1).long()
        r = place["page_table"].gather(1, at).clamp(min=0).long() * sp + pos % place["page"] * st
    else:
        r = (place["cu_L"][:-1, None].long() + pos) * st
    return (r[..., None] + torch.arange(Hkv, device=pos.device) * sh).clamp(max=place["rows"] - 1)


def _rounded_cache(gen, rows, D):
    """4-bit rows of normal K and V, made piece by piece; one row more than the cache has, for what a plain form discards."""
    k4, v4 = (torch.empty((rows + 1, D // 2), dtype=torch.uint8, device=DEV) for _ in range(2))
    ks = torch.empty((rows + 1, D // 32), dtype=torch.uint8, device=DEV)
    vs = torch.empty(rows + 1, dtype=torch.bfloat16, device=DEV)
    step = 1 << 20
    for i in range(0, rows + 1, step):
        n = min(step, rows + 1 - i)
        k4[i:i + n], ks[i:i + n] = _round_k(_normal(gen, (n, D)).float())
        v4[i:i + n], vs[i:i + n] = _round_v(_normal(gen, (n, D)).float())
    return k4, ks, v4, vs


def _own_cache(s, D, kind="e2m1"):
    from paper_2510_26577_amd import cache4
    p = s["place"]
    more = {}
    if kind == "e2m1":
        more = dict(k_row_scale=s["ks"], v_row_scale=s["vs"])
    elif kind == "e4m3":
        more = dict(k_scale=s["k_scale"], v_scale=s["k_scale"])
    return cache4.make_cache(kind={"bf16": cache4.ROWS_BF16, "e4m3": cache4.ROWS_E4M3, "e2m1": cache4.ROWS_E2M1}[kind], k=s["k"], v=s["v"],
                             cu_L=p["cu_L"], page_table=p["page_table"], page_size=p["page"], strides=tuple(x * D for x in p["strides"]), **more)


def _tree(rng, T):
    parent = np.full(T, -1, np.int32)
    depth = np.zeros(T, np.int64)
    for i in range(1, T):
        ok = np.nonzero(depth[:i] < 8)[0]
        parent[i] = int(rng.choice(ok))
        depth[i] = depth[parent[i]] + 1
    return parent


def _masks(parents, words):
    out = []
    for parent in parents:
        rows = []
        for i, p in enumerate(parent):
            rows.append((rows[p] if p >= 0 else 0) | (1 << i))
        out += [[(r >> (64 * w)) & (2 ** 64 - 1) for w in range(words)] for r in rows]
    return np.array(out, np.uint64).view(np.int64)


def _prepare_attn(case, rng, gen):
    Hq, Hkv, D = HEADS[case["heads"]]
    B, L = case["B"], _lengths(case, rng)
    sizes = rng.permutation([max(1, case["T"] - b * (case["T"] // 8) // B) for b in range(B)])
    parents = [_tree(rng, int(t)) for t in sizes]
    cu_T = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n, max_T = int(cu_T[-1]), int(max(sizes))
    s = dict(kind="attn", Hkv=Hkv, G=Hq // Hkv, max_T=max_T, max_L=int(L.max()), scale=1.0 / math.sqrt(D), place=_place(case, rng, L, Hkv),
             cu_T=_dev(cu_T), L=_dev(L), mask=_dev(_masks(parents, 1 + (max_T > 64))), q=_normal(gen, (n, Hq, D)),
             k_tree=_normal(gen, (n, Hkv, D)), v_tree=_normal(gen, (n, Hkv, D)))
    s["k"], s["ks"], s["v"], s["vs"] = _rounded_cache(gen, s["place"]["rows"], D)
    if own:  # a program with fixed buffers fills the argument block once
        from paper_2510_26577_amd import cache4
        s["out"] = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty((n, Hq), dtype=torch.float32, device=DEV)
        s["args"] = cache4.make_attn_args(q=s["q"], k_tree=s["k_tree"], v_tree=s["v_tree"], cache=_own_cache(s, D), anc_mask=s["mask"],
                                          cu_T=s["cu_T"], L=s["L"], max_T=max_T, max_L=s["max_L"], scale=s["scale"], out=s["out"], lse=s["lse"])
        s["ws"] = cache4.attn_workspace(s["args"], DEV)
    return s


def _prepare_store(case, rng, gen):
    Hq, Hkv, D = HEADS[case["heads"]]
    B, T, n_layers = case["B"], case["T"], case["layers"]
    sizes = rng.permutation([max(1, T - b * (T // 8) // B) for b in range(B)])
    cu_T = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n, width = int(cu_T[-1]), min(T, 9) if case["path"] else T
    place = _place(case, rng, [case["L"] + width] * B, Hkv)
    s = dict(kind="store", Hkv=Hkv, width=width, place=place, cu_T=_dev(cu_T), L=_dev(np.full(B, case["L"], np.int32)), n_layers=n_layers,
             k_rows=_normal(gen, (n_layers, n, Hkv, D)), v_rows=_normal(gen, (n_layers, n, Hkv, D)), path=None, path_len=None,
             L_out=torch.zeros(B, dtype=torch.int32, device=DEV))
    if case["path"]:  # the accepted nodes, in ascending order
        lens = [int(rng.integers(1, min(int(t), width) + 1)) for t in sizes]
        path = np.full((B, width), -1, np.int32)
        for b, k in enumerate(lens):
            path[b, :k] = np.sort(rng.choice(int(sizes[b]), k, replace=False))
        s.update(path=_dev(path), path_len=_dev(lens, np.int32))
    rows = place["rows"] * n_layers + 1
    s.update(k=torch.zeros((rows, D // 2), dtype=torch.uint8, device=DEV), v=torch.zeros((rows, D // 2), dtype=torch.uint8, device=DEV),
             ks=torch.zeros((rows, D // 32), dtype=torch.uint8, device=DEV), vs=torch.zeros(rows, dtype=torch.bfloat16, device=DEV))
    # read back: rows of nodes that were not accepted stay as they are
    s.update(k_back=torch.zeros((n_layers * n + 1, Hkv, D), dtype=torch.bfloat16, device=DEV),
             v_back=torch.zeros((n_layers * n + 1, Hkv, D), dtype=torch.bfloat16, device=DEV))
    if own:
        from paper_2510_26577_amd import cache4
        more = dict(cu_T=s["cu_T"], L=s["L"], path=s["path"], path_len=s["path_len"], max_rows=width, cache=_own_cache(s, D), n_layers=n_layers,
                    layer_stride_cache=place["rows"] * D, layer_stride_rows=n * Hkv * D)
        s["store"] = cache4.make_rows_args(k_rows=s["k_rows"], v_rows=s["v_rows"], L_out=s["L_out"], **more)
        s["load"] = cache4.make_rows_args(k_rows=s["k_back"], v_rows=s["v_back"], **more)
    return s


def _newest_rows(s):
    """Rows of q that the newest tokens have, [B, width], and which of them there are."""
    j = torch.arange(s["width"], device=s["L"].device)
    if s["path"] is None:
        return s["cu_T"][:-1, None].long() + j, j < (s["cu_T"][1:] - s["cu_T"][:-1])[:, None]
    return s["cu_T"][:-1, None].long() + s["path"].clamp(min=0), j < s["path_len"][:, None]


def _prepare_weights(case, rng, gen):
    Hq, Hkv, D = HEADS[case["heads"]]
    B, L, T = case["B"], _lengths(case, rng), case["T"]
    cu_T = np.arange(B + 1, dtype=np.int32) * T
    lens = [int(rng.integers(1, case["n"] + 1)) for _ in range(B)]
    path = np.full((B, case["n"]), -1, np.int32)
    for b, k in enumerate(lens):
        path[b, :k] = np.sort(rng.choice(T, k, replace=False))
    ld = int(L.max()) + 24
    s = dict(kind="weights", rows=case["rows"], Hkv=Hkv, G=Hq // Hkv, D=D, width=case["n"], max_L=int(L.max()), scale=1.0 / math.sqrt(D),
             place=_place(case, rng, L, Hkv), cu_T=_dev(cu_T), L=_dev(L), path=_dev(path), path_len=_dev(lens, np.int32),
             q=_normal(gen, (B * T, Hq, D)), first_pos=_dev(L + 1000, np.int32), pos=torch.zeros((B, Hkv, ld), dtype=torch.int32, device=DEV),
             weight=torch.rand((B, Hkv, ld), generator=gen, device=DEV) * 0.01)
    n = s["place"]["rows"]
    if case["rows"] == "e2m1":
        s["k"], s["ks"], s["v"], s["vs"] = _rounded_cache(gen, n, D)
    else:
        s["k"], s["k_scale"] = _normal(gen, (n, D)), 1.0
        if case["rows"] == "e4m3":
            s["k_scale"] = float(s["k"].abs().max()) / 448.0
            s["k"] = (s["k"].float() / s["k_scale"]).to(torch.float8_e4m3fn).view(torch.uint8)
        s["v"] = s["k"]  # (not read)
    # what the attention gave for those rows
    r, there = _newest_rows(s)
    lse = torch.logsumexp(_seen_scores(s), -1).unflatten(-1, (s["width"], s["G"])).permute(0, 2, 1, 3).flatten(2)
    s["lse"] = torch.full((B * T, Hq), 5.0, device=DEV)
    s["lse"][r[there]] = lse[there]
    if own:
        from paper_2510_26577_amd import evict
        s["args"] = evict.make_key_weight_args(q=s["q"], lse=s["lse"], cache=_own_cache(s, D, case["rows"]), cu_T=s["cu_T"], path=s["path"],
                                               path_len=s["path_len"], L=s["L"], max_rows=case["n"], max_L=s["max_L"], scale=s["scale"],
                                               weight=s["weight"], pos=s["pos"], first_pos=s["first_pos"])
    return s


def _weights_of_keys(gen, shape):
    """Accumulated attention: a few keys get most of it, and many have exactly none yet."""
    w = torch.empty(shape, device=DEV).log_normal_(0.0, 2.0, generator=gen)
    return w * (torch.rand(shape, generator=gen, device=DEV) < 0.9)


def _prepare_select(case, rng, gen):
    n_layers, B, H, L = case["layers"], case["B"], case["H"], _lengths(case, rng)
    ld = int(L.max())
    s = dict(kind="select", max_L=ld, first=case["first"], L=_dev(L), keep=_dev(np.full(B, case["keep"], np.int32)),
             newest=_dev(L - case["recent"], np.int32), weight=_weights_of_keys(gen, (n_layers, B, H, ld)), pos=None,
             src=torch.full((n_layers, B, H, case["keep"]), -1, dtype=torch.int32, device=DEV), L_out=torch.zeros(B, dtype=torch.int32, device=DEV))
    if case["aged"]:
        s["pos"] = torch.rand((n_layers, B, H, ld), generator=gen, device=DEV).argsort(-1).to(torch.int32)
    if own:
        from paper_2510_26577_amd import evict
        s["args"] = evict.make_select_args(weight=s["weight"], pos=s["pos"], newest=s["newest"], L=s["L"], keep=s["keep"], max_L=ld,
                                           n_first=s["first"], src=s["src"], L_out=s["L_out"])
    return s


def _prepare_move(case, rng, gen):
    Hq, Hkv, D = HEADS[case["heads"]]
    n_layers, B, L = case["layers"], case["B"], case["L"]
    s = dict(kind="move", rows=case["rows"], Hkv=Hkv, max_L=L, first=4, L=_dev(np.full(B, L, np.int32)), keep=_dev(np.full(B, case["keep"], np.int32)),
             newest=_dev(np.full(B, L - case["keep"] // 4, np.int32)), weight=_weights_of_keys(gen, (n_layers, B, Hkv, L)), pos=None,
             src=torch.full((n_layers, B, Hkv, case["keep"]), -1, dtype=torch.int32, device=DEV), L_out=torch.zeros(B, dtype=torch.int32, device=DEV))
    _plain_select(s)
    s["pos"] = torch.arange(L, dtype=torch.int32, device=DEV).expand(n_layers, B, Hkv, L).contiguous()
    # dense, token-major, every sequence with its room
    s["place"] = dict(page_table=None, cu_L=_dev(np.arange(B + 1) * L, np.int32), page=0, strides=(0, Hkv, 1), rows=B * L * Hkv)
    s["k"], s["v"] = (_normal(gen, (n_layers, B, L, Hkv, D)) for _ in range(2))
    if case["rows"] == "e4m3":
        s["k"], s["v"] = (x.to(torch.float8_e4m3fn) for x in (s["k"], s["v"]))
        s["k_scale"] = 1.0
    if own:
        from paper_2510_26577_amd import evict
        s["args"] = evict.make_move_args(src=s["src"], n=s["L_out"], cache=_own_cache(s, D, case["rows"]), Hkv=Hkv, D=D, max_keep=case["keep"],
                                         weight=s["weight"], pos=s["pos"], layer_stride_cache=s["place"]["rows"] * D)
    return s


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    make = {"attn": _prepare_attn, "store": _prepare_store, "weights": _prepare_weights, "select": _prepare_select, "move": _prepare_move}
    return make[case["kind"]](case, rng, gen)


# ---- the plain forms ----
def _plain_attn(s):
    B, Hkv, G, max_T, max_L = s["L"].shape[0], s["Hkv"], s["G"], s["max_T"], s["max_L"]
    dev = s["L"].device
    t, i = torch.arange(max_L, device=dev), torch.arange(max_T, device=dev)
    at = _row_numbers(s["place"], t.expand(B, -1), Hkv)
    sizes = s["cu_T"][1:] - s["cu_T"][:-1]
    node = (s["cu_T"][:-1, None].long() + i).clamp(max=s["q"].shape[0] - 1)  # [B, max_T], those past a tree's end are masked
    K = torch.cat([_k_values(s["k"][at], s["ks"][at]), s["k_tree"][node].float()], 1).transpose(1, 2)  # [B, Hkv, max_L + max_T, D]
    q = s["q"][node].float().unflatten(2, (Hkv, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B, Hkv, max_T * G, D]
    x = torch.matmul(q, K.transpose(2, 3).contiguous()) * s["scale"]
    del K
    bits = (s["mask"][node][:, :, i // 64] >> (i % 64)) & 1
    seen = torch.cat([(t < s["L"][:, None])[:, None].expand(-1, max_T, -1), (bits != 0) & (i < sizes[:, None])[:, None]], 2)
    x.masked_fill_(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    V = torch.cat([_v_values(s["v"][at], s["vs"][at]), s["v_tree"][node].float()], 1).transpose(1, 2).contiguous()
    out = torch.matmul(x, V) / torch.where(total == 0, 1.0, total)
    ragged = lambda y: y.unflatten(2, (max_T, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # noqa: E731  [B, max_T, Hq, ..]
    b = torch.searchsorted(s["cu_T"][1:].contiguous(), torch.arange(s["q"].shape[0], device=dev, dtype=torch.int32), right=True)
    j = torch.arange(s["q"].shape[0], device=dev) - s["cu_T"][b]
    lse = (top + torch.log(total))
    return ragged(out)[b, j].to(torch.bfloat16), ragged(lse)[b, j][..., 0]


def _plain_store(s):
    Hkv, n = s["Hkv"], s["k_rows"].shape[1]
    r, there = _newest_rows(s)
    pos = s["L"][:, None].long() + torch.arange(s["width"], device=r.device)
    layer = torch.arange(s["n_layers"], device=r.device)[:, None, None]
    spare, spare_row = s["k"].shape[0] - 1, s["k_back"].shape[0] - 1  # rows that no sequence has go there
    to = torch.where(there[None, ..., None], _row_numbers(s["place"], pos, Hkv) + layer[..., None] * s["place"]["rows"], spare)
    back = torch.where(there, r + layer * n, spare_row)
    r = r.clamp(max=n - 1)
    s["k"][to], s["ks"][to] = _round_k(s["k_rows"][:, r].float())
    s["v"][to], s["vs"][to] = _round_v(s["v_rows"][:, r].float())
    s["L_out"].copy_(s["L"] + there.sum(1))
    s["k_back"][back] = _k_values(s["k"][to], s["ks"][to]).to(torch.bfloat16)
    s["v_back"][back] = _v_values(s["v"][to], s["vs"][to]).to(torch.bfloat16)


def _seen_scores(s):
    """Scaled scores of the newest tokens' rows, -inf where a position lies behind the row's own: [B, Hkv, width * G, max_L]."""
    t = torch.arange(s["max_L"], device=s["L"].device)
    r, there = _newest_rows(s)
    at = _row_numbers(s["place"], t.expand(r.shape[0], -1), s["Hkv"])
    if s["rows"] == "e2m1":
        K = _k_values(s["k"][at], s["ks"][at])
    elif s["rows"] == "e4m3":
        K = s["k"].view(torch.float8_e4m3fn)[at].float() * s["k_scale"]
    else:
        K = s["k"][at].float()
    q = s["q"][r.clamp(max=s["q"].shape[0] - 1)].float().unflatten(2, (s["Hkv"], s["G"])).permute(0, 2, 1, 3, 4).flatten(2, 3)
    x = torch.matmul(q, K.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    own_pos = (s["L"] - s["path_len"])[:, None] + torch.arange(s["width"], device=t.device)
    seen = (t <= own_pos[..., None]) & there[..., None]
    return x.masked_fill_(~seen.repeat_interleave(s["G"], 1)[:, None], -math.inf)


def _plain_weights(s):
    r, there = _newest_rows(s)
    lse = s["lse"][r.clamp(max=s["q"].shape[0] - 1)].unflatten(2, (s["Hkv"], s["G"])).permute(0, 2, 1, 3).flatten(2)
    add = torch.exp(_seen_scores(s) - lse[..., None]).sum(2)
    t = torch.arange(s["max_L"], device=r.device)
    old, first = (t < s["L"][:, None])[:, None], (s["L"] - s["path_len"])[:, None]
    w, p = s["weight"][..., :s["max_L"]], s["pos"][..., :s["max_L"]]
    w.copy_(torch.where(old, torch.where((t < first)[:, None], w, 0.0) + add, w))
    p.copy_(torch.where(((t >= first) & (t < s["L"][:, None]))[:, None], (s["first_pos"][:, None] + t - first)[:, None], p))


def _plain_select(s):
    w = s["weight"]
    t = torch.arange(s["max_L"], device=w.device)
    age = t if s["pos"] is None else s["pos"]
    here = (t < s["L"][:, None])[:, None]
    safe = (t < s["first"]) | (age >= s["newest"][:, None, None])
    key = torch.where(here, torch.where(safe, math.inf, w), -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]
    n = torch.minimum(s["keep"], s["L"])
    kept = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, order, (t < n[:, None])[:, None].expand_as(order))
    low = (t < n[:, None])[:, None]
    gap, late = ~kept & low, kept & ~low
    rank = torch.where(late, late.cumsum(-1) - 1, s["max_L"])
    fill = torch.zeros((*key.shape[:-1], s["max_L"] + 1), dtype=torch.int64, device=w.device).scatter_(-1, rank, t.expand_as(rank))
    src = torch.where(gap, fill.gather(-1, (gap.cumsum(-1) - 1).clamp(min=0)), t)
    m = min(s["src"].shape[-1], s["max_L"])
    s["src"][..., :m] = torch.where(low[..., :m], src[..., :m].to(torch.int32), s["src"][..., :m])
    s["L_out"].copy_(n)


def _plain_move(s):
    m, dev = s["src"].shape[-1], s["L"].device
    j = torch.arange(m, device=dev)
    there = (j < s["L_out"][:, None])[:, None]
    old = torch.where(there & (s["src"] >= 0), s["src"], j).long()  # [layers, B, Hkv, m]; entries past n move nothing
    for x in (s["k"], s["v"]):
        rows = x.view(torch.uint8) if x.element_size() == 1 else x
        rows = rows.permute(0, 1, 3, 2, 4)
        rows[..., :m, :] = rows.gather(3, old[..., None].expand(-1, -1, -1, -1, rows.shape[-1]))
    for x in (s["weight"], s["pos"]):
        x[..., :m] = x.gather(-1, old)


def _results(s):
    if s["kind"] == "store":
        return s["k_back"][:-1], s["v_back"][:-1], s["L_out"]
    if s["kind"] == "weights":
        return s["weight"], s["pos"]
    if s["kind"] == "select":
        return s["src"], s["L_out"]
    return s["k"], s["v"], s["weight"], s["pos"]


def run(state):
    s = state
    if not own:
        if s["kind"] == "attn":
            return _plain_attn(s)
        {"store": _plain_store, "weights": _plain_weights, "select": _plain_select, "move": _plain_move}[s["kind"]](s)
        return _results(s)
    from paper_2510_26577_amd import cache4, evict
    if s["kind"] == "attn":
        cache4.tree_verify_attn_raw(s["args"])
        return s["out"], s["lse"]
    if s["kind"] == "store":
        cache4.store_raw(s["store"])
        cache4.load_raw(s["load"])
    else:
        {"weights": evict.key_weights_raw, "select": evict.select_raw, "move": evict.move_raw}[s["kind"]](s["args"])
    return _results(s)


# ---- the definitions in 64 bits, sequence by sequence ----
def _exact_codes(x):
    x = x.to(torch.int64)
    c = torch.stack([x & 15, x >> 4], -1).flatten(-2)
    e, m = (c >> 1) & 3, (c & 1).double()
    v = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e - 1).double())
    return torch.where(c >= 8, -v, v)


def _exact_rows(s, b, n, which):
    """The values of sequence b's first n positions, [n, Hkv, D]."""
    place, Hkv = s["place"], s["Hkv"]
    t = torch.arange(n, device=DEV)
    if place["page"]:
        base = place["page_table"][b].long()[t // place["page"]] * place["strides"][0] + t % place["page"] * place["strides"][1]
    else:
        base = (int(place["cu_L"][b]) + t) * place["strides"][1]
    r = base[:, None] + torch.arange(Hkv, device=DEV) * place["strides"][2]
    kind = s.get("rows", "e2m1")
    if kind == "bf16":
        return s[which][r].double()
    if kind == "e4m3":
        return s[which].view(torch.float8_e4m3fn)[r].double() * s["k_scale"]
    v = _exact_codes(s[which][r])
    if which == "k":
        return v * (2.0 ** (s["ks"][r].double() - 127)).repeat_interleave(32, -1)
    return v * s["vs"][r].double()[..., None]


def _exact_attn(s):
    outs, lses = [], []
    cu, G = s["cu_T"].tolist(), s["G"]
    for b, L in enumerate(s["L"].tolist()):
        lo, hi = cu[b], cu[b + 1]
        K = torch.cat([_exact_rows(s, b, L, "k"), s["k_tree"][lo:hi].double()])
        V = torch.cat([_exact_rows(s, b, L, "v"), s["v_tree"][lo:hi].double()])
        words = s["mask"][lo:hi].cpu().numpy().view(np.uint64)
        ok = torch.ones((hi - lo, L + hi - lo), dtype=torch.bool)
        for j in range(hi - lo):
            ok[:, L + j] = torch.from_numpy(((words[:, j // 64] >> np.uint64(j % 64)) & np.uint64(1)).astype(bool))
        ok = ok.to(DEV)
        o, l = [], []
        for h in range(s["Hkv"] * G):
            x = (s["q"][lo:hi, h].double() @ K[:, h // G].T) * s["scale"]
            x = torch.where(ok, x, -math.inf)
            z = torch.logsumexp(x, 1)
            o.append(torch.exp(x - z[:, None]) @ V[:, h // G])
            l.append(z)
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(l, 1))
    return torch.cat(outs), torch.cat(lses)


def _exact_rounding(x, s):
    """Nearest code's value, the even code of two."""
    codes = [0, 2, 4, 6, 1, 3, 5, 7]
    far = torch.stack([(x.abs() - _MAGNITUDES[c] * s).abs() for c in codes])
    near = torch.tensor([_MAGNITUDES[c] for c in codes], dtype=torch.float64, device=x.device)[far.argmin(0)] * s
    return torch.where(x < 0, -near, near)


def _exact_store(s):
    k, v = torch.zeros_like(s["k_back"][:-1], dtype=torch.float64), torch.zeros_like(s["v_back"][:-1], dtype=torch.float64)
    n, cu, lens = s["k_rows"].shape[1], s["cu_T"].tolist(), []
    for b in range(len(cu) - 1):
        nodes = list(range(cu[b], cu[b + 1])) if s["path"] is None else [cu[b] + i for i in s["path"][b, :int(s["path_len"][b])].tolist()]
        lens.append(len(nodes))
        for layer in range(s["n_layers"]):
            x = s["k_rows"][layer, nodes].double().unflatten(-1, (-1, 32))
            a = x.abs().amax(-1, keepdim=True)
            m, e = torch.frexp(a / 6)
            k[[layer * n + i for i in nodes]] = _exact_rounding(x, 2.0 ** torch.where(m == 0.5, e - 1, e).double()).flatten(-2)
            x = s["v_rows"][layer, nodes].double()
            m, e = torch.frexp(x.abs().amax(-1, keepdim=True) / 6)
            v[[layer * n + i for i in nodes]] = _exact_rounding(x, torch.ceil(m * 16) / 16 * 2.0 ** e.double())
    return k, v, s["L"] + torch.tensor(lens, dtype=torch.int32, device=DEV)


def _exact_weights(s):
    w, p = s["weight"].double(), s["pos"].clone()
    cu = s["cu_T"].tolist()
    for b, L in enumerate(s["L"].tolist()):
        nodes = [cu[b] + i for i in s["path"][b, :int(s["path_len"][b])].tolist()]
        n = len(nodes)
        K = _exact_rows(s, b, L, "k")
        w[b, :, L - n:L] = 0.0
        p[b, :, L - n:L] = s["first_pos"][b] + torch.arange(n, device=DEV, dtype=torch.int32)
        for i, node in enumerate(nodes):
            end = L - n + i + 1
            for g in range(s["Hkv"]):
                h = slice(g * s["G"], (g + 1) * s["G"])
                x = (s["q"][node, h].double() @ K[:end, g].T) * s["scale"] - s["lse"][node, h].double()[:, None]
                w[b, g, :end] += torch.exp(x).sum(0)
    return w, p


def _exact_move(s):
    new = [x.double() for x in (s["k"], s["v"], s["weight"])] + [s["pos"].clone()]
    for layer in range(s["src"].shape[0]):
        for b, n in enumerate(s["L_out"].tolist()):
            for h in range(s["Hkv"]):
                old = s["src"][layer, b, h, :n].long()
                for to, x in zip(new[:2], (s["k"], s["v"])):
                    to[layer, b, :n, h] = x[layer, b, :, h].double()[old]
                for to, x in zip(new[2:], (s["weight"], s["pos"])):
                    to[layer, b, h, :n] = x[layer, b, h, old].to(to.dtype)
    return new


def exact(case, seed):
    """(A choice of slots has no other value than the plain form's.)"""
    if case["kind"] == "select":
        return None
    s = prepare(case, seed)
    return {"attn": _exact_attn, "store": _exact_store, "weights": _exact_weights, "move": _exact_move}[case["kind"]](s)


# ---- what a pass cannot do without ----
def work(case):
    B = case["B"]
    if case["kind"] == "select":
        L = 0.5 * (case["L_lo"] + case["L_hi"]) if B > 1 else case["L_hi"]
        n = case["layers"] * B * case["H"]
        return {"bytes": n * (L * (8 if case["aged"] else 4) + min(L, case["keep"]) * 4), "flops": n * L}
    Hq, Hkv, D = HEADS[case["heads"]]
    row = D // 2 + D // 32 + D // 2 + 2  # K and V of one head in 4 bits
    if case["kind"] == "move":
        n, keep = case["layers"] * B * Hkv, min(case["L"], case["keep"])
        moved = keep * (1 - keep / case["L"]) * 0.7  # about: the newest quarter lies behind
        return {"bytes": n * (keep * 4 + moved * 2 * (2 * D * (2 if case["rows"] == "bf16" else 1) + 8)), "flops": n * keep}
    if case["kind"] == "store":
        rows = case["layers"] * B * Hkv * (0.5 * (min(case["T"], 9) + 1) if case["path"] else case["T"])
        return {"bytes": rows * 2 * (4 * D + row), "flops": rows * 2 * D}
    L = case["L_hi"] if B == 1 else 0.5 * (case["L_lo"] + case["L_hi"])
    if case["kind"] == "attn":
        T = case["T"]
        return {"bytes": B * (L * Hkv * row + T * Hkv * D * 4 + T * Hq * (D * 4 + 4)), "flops": 4.0 * B * T * Hq * D * (L + T)}
    n = 0.5 * (1 + case["n"])
    one = {"bf16": 2 * D, "e4m3": D, "e2m1": D // 2 + D // 32}[case["rows"]]
    return {"bytes": B * (L * Hkv * (one + 8) + n * Hq * (2 * D + 4)), "flops": 2.0 * B * n * Hq * D * L}
