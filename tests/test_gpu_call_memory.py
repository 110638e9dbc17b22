"""What the Python calls make for themselves and their callers when they are queued on another stream than the current one: memory that no other
work has or gets."""
import numpy as np
import pytest

from tests import cache_cases as cc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _calls(torch):
    """name -> a call on tensors that live on, given its stream; its results."""
    from paper_2510_26577_amd import binding, cache4, chunk, draft, evict, rotary, verify, workloads as wl
    Hq, Hkv, D, n = 8, 2, 64, 40
    x = torch.randn((n, Hq + 2 * Hkv, D), device="cuda").bfloat16()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    freq, cu, zero = cc.dev(rotary.frequencies(D)[0]), cc.dev([0, n], np.int32), cc.dev([0], np.int32)
    rows = [torch.zeros((600, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    room = cc.dev([0, 600], np.int32)
    cache = cache4.make_cache(kind=0, k=rows[0], v=rows[1], cu_L=room)
    four = cache4.make_cache(kind=2, k=torch.zeros((600, Hkv, D // 2), dtype=torch.uint8, device="cuda"), v=torch.zeros((600, Hkv, D // 2), dtype=torch.uint8, device="cuda"),
                             k_row_scale=torch.full((600 * Hkv, D // 32), 120, dtype=torch.uint8, device="cuda"),
                             v_row_scale=torch.ones(600 * Hkv, dtype=torch.bfloat16, device="cuda"), cu_L=cc.dev([0, 600], np.int32))
    L, keep, cu5 = cc.dev([500], np.int32), cc.dev([200], np.int32), cc.dev([0, 5], np.int32)
    place = dict(cu_T=cu, L=zero, freq=freq, dims=D)
    packed = [t.contiguous() for t in (q, k, v)]
    mask = cc.dev(cc.mask_words(np.tril(np.ones((n, n), bool)), 1))
    weight = torch.rand((1, Hkv, 500), device="cuda")
    parts = torch.randn((3, n, D), device="cuda"), torch.randn((3, n), device="cuda")
    score, logp = torch.zeros(5, device="cuda"), torch.log_softmax(torch.randn((5, 2000), device="cuda"), -1)
    chance = torch.sort(torch.rand((2, 100), device="cuda"), descending=True)[0]
    cost = torch.cumsum(torch.full((100,), 0.05, dtype=torch.float64, device="cuda"), 0) + 1.0
    rng = np.random.Generator(np.random.PCG64(31))
    tree, count = wl.tree_expand_prune(rng, n).astype(np.int32), np.array([0, n], np.int32)
    p, r, tok, u, uf = wl.sampling_inputs(rng, tree, count, 20000, drift=0.6)
    parent, tokens = cc.dev(tree), cc.dev(tok, np.int32)
    sample = [parent, cu, tokens, *(cc.dev(x, np.float32) for x in (p, r, u, uf))]
    scores, heads = torch.rand((16, 145), device="cuda"), cc.dev([0, n // 2], np.int32)
    node_score = torch.sort(torch.rand(n, device="cuda"), descending=True)[0]
    return {
        "verify": lambda s: binding.tree_verify_attn(*packed, *rows, None, cu, L, max_T=n, max_L=500, scale=0.1, cu_L=room, parent=parent, num_splits=8, stream=s),
        "masks": lambda s: (binding.build_ancestor_mask(parent, cu, n, stream=s),),
        "greedy": lambda s: verify.accept_greedy(parent, cu, tokens, tokens, 9, stream=s),
        "sampling": lambda s: verify.accept_sampling(*sample, 9, stream=s),
        "rerank": lambda s: draft.rerank_count(scores, cost, 72, 1.0, stream=s),
        "subtree": lambda s: draft.select_subtree(node_score, parent, cu, heads, n, total_kept=n // 2, stream=s),
        "rotate": lambda s: rotary.rotate(q=q, k=k, stream=s, **place),
        "append": lambda s: (rotary.append(q=q, k=k, v=v, cache=cache, stream=s, **place),),
        "attn": lambda s: chunk.attn(packed[0], cache, cu, L, Hkv=Hkv, max_T=n, max_L=500, scale=0.1, num_splits=3, stream=s),
        "attn 4 bit": lambda s: cache4.tree_verify_attn(*packed, four, cu, L, max_T=n, max_L=500, scale=0.1, anc_mask=mask, num_splits=3, stream=s),
        "select": lambda s: evict.select(weight, L, keep, max_L=500, max_keep=200, stream=s),
        "merge": lambda s: binding.merge_splits(*parts, stream=s),
        "expand": lambda s: draft.expand_layer(cu5, score, logp, 8, 5, stream=s),
        "breadth": lambda s: draft.breadth_count(chance, cost, 1.0, 1.0, stream=s),
    }


@pytest.fixture(scope="module")
def calls(torch):
    return _calls(torch)


NAMES = ["verify", "masks", "greedy", "sampling", "rerank", "subtree", "rotate", "append", "attn", "attn 4 bit", "select", "merge", "expand", "breadth"]


def _same(a, b):
    import torch
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


def _places(tensors):
    return {t.untyped_storage().data_ptr() for t in tensors}


def _like(tensors):
    import torch
    return [torch.empty(t.untyped_storage().nbytes(), dtype=torch.uint8, device="cuda") for t in tensors for _ in range(3)]


@pytest.mark.parametrize("name", NAMES)
def test_results_on_another_stream_are_the_same(torch, calls, name):
    want = [t.clone() for t in calls[name](None)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = calls[name](s)
    torch.cuda.synchronize()
    assert _same(got, want)
    other = type("Handle", (), dict(cuda_stream=s.cuda_stream))()  # anything that names a stream
    got = calls[name](other)
    torch.cuda.synchronize()
    assert _same(got, want)


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_works_on_is_not_taken(torch, calls, name):
    """Freed on the current stream, whose work on it waits: a call queued elsewhere gets other memory."""
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = _like(calls[name](None))
    torch.cuda.synchronize()
    torch.cuda._sleep(5_000_000)
    for t in freed:
        t.fill_(255)
    places = _places(freed)
    del freed, t
    got = calls[name](s)
    assert not places & _places(got)
    torch.cuda.synchronize()
    assert _same(got, calls[name](None))


@pytest.mark.parametrize("name", NAMES)
def test_results_that_are_dropped_are_not_handed_out_while_their_stream_works(torch, calls, name):
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(5_000_000)
    got = calls[name](s)
    places = _places(got)
    new = _like(got)
    del got
    new += _like(new)
    assert not places & _places(new)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_results_that_are_dropped_behind_their_use_are_not_written_before_it(torch, calls, name):
    """Used on the current stream, which waits for the call's; then the next call on that stream, which does not wait for the use."""
    s, here = torch.cuda.Stream(), torch.cuda.current_stream()
    want = [t.clone() for t in calls[name](None)]
    torch.cuda.synchronize()
    got = calls[name](s)
    here.wait_stream(s)
    torch.cuda._sleep(5_000_000)
    used = [t.clone() for t in got]
    places = _places(got)
    del got
    again = calls[name](s)
    assert not places & _places(again)
    torch.cuda.synchronize()
    assert _same(used, want) and _same(again, want)


@pytest.mark.parametrize("name", NAMES)
def test_calls_on_a_second_stream_of_a_capture(torch, calls, name):
    """Queued on a stream that forks off the captured one: replays, with eager calls and other memory between them, give the eager result."""
    want = [t.clone() for t in calls[name](None)]
    s, fork, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        fork.wait_stream(s)
        got = calls[name](fork)
        s.wait_stream(fork)
        more = [torch.zeros_like(t) for t in got]  # (would take memory that the call has let go)
    for _ in range(3):
        for t in got:
            t.zero_()
        other = _like(got)
        for t in other:
            t.fill_(255)
        eager = calls[name](None)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(got, want) and _same(eager, want) and not any(bool(t.any()) for t in more)
        del other, eager
