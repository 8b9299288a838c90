"""Registers and LDS of the cache operators' kernels (the metadata of the built library): nothing spills vector registers, and as many workgroups
fit on a CU as the host's rules for splits and steps count on."""
import pytest

from paper_2605_23200_amd import binding as B
from test_kernel_resources import _kernels

LDS = 160 * 1024


@pytest.fixture(scope="module")
def kernels():
    B.lib()
    return _kernels(B.LIB_PATH)


def _of(kernels, name):
    return {args: k for n, args, k in kernels if n == name}


def _fit(k, lds=0):
    """Workgroups of four waves on a CU: one wave each on the four SIMDs, of 512 registers in steps of 8."""
    return min(512 // (-(-k[".vgpr_count"] // 8) * 8), LDS // (k[".group_segment_fixed_size"] + lds) if k[".group_segment_fixed_size"] + lds else 99)


@pytest.mark.parametrize("name,count", [("attend_kernel", 24), ("attend_pair_kernel", 5), ("attend_join_kernel", 4), ("attend_weights_kernel", 12),
                                        ("append_kernel", 32), ("move_kernel", 2), ("pages_kernel", 1)])
def test_nothing_spills(kernels, name, count):
    found = _of(kernels, name)
    assert len(found) == count
    assert {a: k[".vgpr_spill_count"] for a, k in found.items() if k[".vgpr_spill_count"]} == {}


def test_recode_does_not_spill(kernels):
    assert {a: k[".vgpr_spill_count"] for a, k in _of(kernels, "recode_kernel").items() if k[".vgpr_spill_count"]} == {}


def test_attention_head_by_head(kernels):
    """Three workgroups on a CU, two with more than 16 queries, one fewer with fp32 queries over 128 channels."""
    for (el, bf16, dim, tiles), k in _of(kernels, "attend_kernel").items():
        assert _fit(k) >= (3 if tiles == 1 else 2) - (not bf16 and dim == 128), (el, bf16, dim, tiles)


def test_attention_two_heads_at_a_time(kernels):
    """Two: one round is one on a CU, and batches above it share CUs."""
    for args, k in _of(kernels, "attend_pair_kernel").items():
        assert _fit(k) >= 2, args


def test_weights_from_keys_again(kernels):
    """Four workgroups of bf16 queries, two of fp32, with the operands of 32 queries in LDS."""
    for (el, bf16, dim), k in _of(kernels, "attend_weights_kernel").items():
        group = 2 * (dim // 32) * (1 if bf16 else 3) * 64 * 16
        assert _fit(k, group) >= (4 if bf16 else 2), (el, bf16, dim)


def test_append_and_pages(kernels):
    """append: three workgroups where keys are formed in 64 bits, else four; pages: six."""
    for (el, bf16, dim, any_halves), k in _of(kernels, "append_kernel").items():
        assert _fit(k) >= (3 if el >= B.INT8 else 4), (el, bf16, dim, any_halves)
    assert _fit(_of(kernels, "pages_kernel")[()]) >= 6
