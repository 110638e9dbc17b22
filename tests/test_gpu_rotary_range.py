"""GPU tests of tva_rotate: norms of heads far from 1, where an element times its weight lies outside fp32 before it is normed."""
import numpy as np
import pytest

from oracle import cache_oracle, layer_oracle as orc
from tests import cache_cases as cc
from tests.test_gpu_rotary import check

pytestmark = pytest.mark.gpu
bf16, to_bf16 = cache_oracle.bf16, cache_oracle.to_bf16


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _normed(torch, x, w, dims, interleaved, eps):
    from paper_2510_26577_amd import rotary
    pos = [0, 5, 7000][:len(x)]
    freq, _ = rotary.frequencies(max(dims, 4))
    out, _ = rotary.rotate(q=cc.dev(x), q_norm=cc.dev(w), pos=cc.dev(pos, np.int32), freq=cc.dev(freq), dims=dims, interleaved=interleaved, eps=eps)
    torch.cuda.synchronize()
    return bf16(cc.bits(out)), orc.heads(bf16(x), pos, freq[:dims // 2], dims, interleaved, 1.0, bf16(w), eps)


@pytest.mark.parametrize("D,dims,interleaved", [(64, 64, False), (128, 64, True), (128, 128, False), (128, 0, False)])
@pytest.mark.parametrize("heads,weights,eps", [(2.0 ** 58, 2.0 ** 75, 1e-6), (2.0 ** -58, 2.0 ** -85, 0.0), (2.0 ** -40, 2.0 ** 20, 1e-6), (2.0 ** 58, 2.0 ** -60, 0.0)])
def test_heads_and_weights_far_from_one(torch, D, dims, interleaved, heads, weights, eps):
    """(Sums of squares are within fp32: 128 * 2^120 at most, 2^-130 at least.)"""
    rng = np.random.default_rng(D + dims)
    x = to_bf16(np.clip(rng.standard_normal((3, 3, D)), -2, 2) * heads)
    w = to_bf16((1 + 0.3 * np.clip(rng.standard_normal(D), -2, 2)) * weights)
    got, (want, size) = _normed(torch, x, w, dims, interleaved, eps)
    check(got, want, size)


@pytest.mark.parametrize("D,dims,interleaved", [(64, 64, False), (128, 64, True), (128, 128, False), (128, 0, False)])
def test_heads_whose_squares_are_past_the_range_become_zero(torch, D, dims, interleaved):
    rng = np.random.default_rng(D)
    x = rng.standard_normal((3, 2, D))
    x[0, 0] *= 2.0 ** 125 / np.abs(x[0, 0]).max()  # times weights up to 16: past 2^128
    x[1, 1] = 2.0 ** 61 * np.sign(x[1, 1])          # 64 or 128 times 2^122
    w = to_bf16(rng.uniform(8, 16, D))
    got, (want, size) = _normed(torch, to_bf16(x), w, dims, interleaved, 1e-6)
    assert (got[0, 0] == 0).all() and (got[1, 1] == 0).all()
    for at in [(0, 1), (1, 0), (2, 0), (2, 1)]:
        check(got[at][None], want[at][None], size[at][None])
