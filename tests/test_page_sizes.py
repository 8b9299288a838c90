"""Sizes that ams_assign_pages refuses, on the host: nothing is launched.  (Its kernel counts stretches of tables and of slots in 32 bits.)"""
import pytest

from paper_2605_23200_amd import binding as B
from test_cache4 import _pages
from test_cache_abi import _p


@pytest.mark.parametrize("kw", [
    dict(max_blocks_per_seq=(1 << 30) + 1), dict(max_blocks_per_seq=2 ** 31 - 1), dict(max_blocks_per_seq=2 ** 31 - 127),
    dict(n_slots=(1 << 36) + 1), dict(n_slots=2 ** 63 - 1), dict(n_slots=2 ** 63 - 64)])
def test_tables_and_slots_beyond_what_is_counted(kw):
    assert _pages(_p(), **kw) == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("batch,kw", [(300, dict(max_blocks_per_seq=1 << 30)), (3, dict(max_blocks_per_seq=1 << 30, n_slots=(1 << 36) + 1)),
                                      (130, dict(max_blocks_per_seq=1 << 30, n_slots=1 << 36))])
def test_together_too_many(batch, kw):
    assert _pages(_p(n_layers=1, batch=batch, n_kv_heads=1), **kw) == B.ERR_UNSUPPORTED


def test_batches():
    assert _pages(_p(batch=(1 << 20) + 1, t_max=16, t_stride=16)) == B.ERR_UNSUPPORTED
    assert _pages(_p(batch=-1)) == B.ERR_INVALID_ARG and _pages(_p(t_max=0)) == B.ERR_INVALID_ARG
    assert _pages(_p(t_max=(1 << 30) + 1, batch=1), max_blocks_per_seq=1 << 30) == B.ERR_UNSUPPORTED
