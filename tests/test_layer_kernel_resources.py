"""What the compiler gave the kernels of include/tva_layer.h: registers for the workgroups that share a compute unit, nothing spilled where
rows are found by scalar addresses (CPU: the built library's own kernel descriptors)."""
import pytest

from tests.test_kernel_resources import kernels


@pytest.fixture(scope="module")
def table():
    t = {n: k for n, k in kernels().items() if "chunk_kernel" in n or "rotate_kernel" in n}
    assert sum("chunk_kernel" in n for n in t) == 72 and sum("rotate_kernel" in n for n in t) == 32, len(t)
    return t


def test_two_workgroups_of_four_waves_or_one_of_eight_fit_a_compute_unit(table):
    for name, k in table.items():
        if "chunk_kernel" in name:
            assert k[".vgpr_count"] <= 256, name
            assert k[".group_segment_fixed_size"] <= (160 if "ELi8ELi1ELi2E" in name else 80) * 1024, name


def test_chunks_in_sequences_and_whole_pages_spill_nothing(table):
    """(The last two arguments: how rows are found, 2 being row by row, and whether it is a tree.)"""
    seen = 0
    for name, k in table.items():
        if "chunk_kernel" in name and ("ELi0ELb0E" in name or "ELi1ELb0E" in name):
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, (name, k[".vgpr_spill_count"])
            seen += 1
    assert seen == 24


def test_rotary_kernels_leave_registers_for_many_waves(table):
    for name, k in table.items():
        if "rotate_kernel" in name:
            assert k[".vgpr_spill_count"] == 0 and k[".vgpr_count"] <= 96, (name, k[".vgpr_count"])
