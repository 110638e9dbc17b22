"""How many query rows a workgroup of the attention over 4-bit rows takes (CPU: the plan shows in the splits and the workspace)."""
import pytest

from paper_2510_26577_amd import binding, cache4


def _plan(nodes, rows, heads=(32, 8, 128), B=4, max_L=32768):
    a = cache4.Attn4Args()
    a.B, a.max_L, a.max_T, a.sum_T, a.mask_words, a.scale, a.plan_rows = B, max_L, nodes, B * nodes, 2, 0.1, rows
    a.Hq, a.Hkv, a.D = heads
    return cache4.plan_splits(a), cache4.workspace_bytes(a)


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        binding.build_library()
    return cache4._lib()


@pytest.mark.parametrize("nodes,rows", [(8, 32), (16, 64), (24, 32), (32, 128), (40, 64), (48, 64), (56, 64), (64, 128), (66, 64), (72, 64), (80, 64), (96, 128),
                                        (100, 64), (112, 64), (128, 128)])
def test_rows_divide_the_row_groups(nodes, rows):
    """Long sequences, four heads to a KV head: at most one wave of a tree's row groups of 32 is idle."""
    plans = {r: _plan(nodes, r) for r in (32, 64, 128)}
    assert _plan(nodes, 0) == plans[rows]
    assert len(set(plans.values())) == 3 or nodes <= 16  # (else nothing is seen)
    groups = -(-nodes // 8)
    assert -(-groups * 32 // rows) * rows - groups * 32 <= 32


def test_little_work_takes_32_rows():
    for nodes in (24, 60, 72, 100):
        assert _plan(nodes, 0, B=1, max_L=2048) == _plan(nodes, 32, B=1, max_L=2048)
