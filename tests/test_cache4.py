"""Caches of 4 bits and pages, on the host: what the entry points refuse before anything is launched, and the definition that the GPU tests go by."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_23200_amd import binding as B
from micro_util import LEVELS, pack_rows, power, values
from test_cache_abi import PTR, _append, _attend, _dense, _evict, _p, _paged, _recode, _tokens


def _micro(**kw):
    return _dense(dtype=B.E2M1, **kw)


def test_types_are_taken_where_8_bits_are():
    p = _p()
    need = B.ams_attend_workspace_bytes(p)
    assert _attend(p, _micro(), n=need - 1) == B.ERR_WORKSPACE_TOO_SMALL          # past the checks of the cache
    assert _attend(p, _paged(dtype=B.E2M1), n=need - 1) == B.ERR_WORKSPACE_TOO_SMALL
    assert _evict(p, _micro(), _micro(base=1 << 20), n=B.ams_evict_workspace_bytes(p) - 1) == B.ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("cache,status", [
    (_micro(base=None), B.ERR_INVALID_ARG), (_micro(base=PTR + 8), B.ERR_INVALID_ARG), (_micro(cap=999), B.ERR_INVALID_ARG),
    (_micro(k_scale=None), B.ERR_INVALID_ARG), (_micro(v_scale=None), B.ERR_INVALID_ARG), (_micro(k_scale=PTR + 4), B.ERR_INVALID_ARG),
    (_micro(v_scale=PTR + 8), B.ERR_INVALID_ARG), (_dense(dtype=5), B.ERR_INVALID_ARG),
    (_paged(dtype=B.E2M1, slots=160008), B.ERR_INVALID_ARG), (_paged(dtype=B.E2M1, block=32), B.ERR_UNSUPPORTED)])
def test_bad_caches(cache, status):
    assert _attend(_p(), cache) == status and _append(_p(), cache, _tokens()) == status
    assert _recode(_p(), cache, _dense(base=1 << 20)) == status and _recode(_p(), _dense(base=1 << 20), cache) == status
    assert _evict(_p(), cache, _dense(base=1 << 20)) == status


def test_in_place_is_refused():
    p = _p()
    assert _recode(p, _micro(), _micro()) == B.ERR_INVALID_ARG and _evict(p, _micro(), _micro()) == B.ERR_INVALID_ARG


def _pages(p, from_=PTR, to=2 * PTR, lens_out=3 * PTR, starts=4 * PTR, slots=5 * PTR, n_slots=10, **kw):
    d = dict(table=PTR, table_out=PTR, max_blocks_per_seq=63, n_pages=100, ring=PTR, state=PTR, state_out=2 * PTR)
    d.update(kw)
    x = B.Pages(*d.values())
    return B.lib().ams_assign_pages(C.byref(p), C.byref(x), from_, to, lens_out, starts, slots, n_slots, None)


@pytest.mark.parametrize("kw", [
    dict(from_=None), dict(to=None), dict(table=None), dict(table_out=None), dict(ring=None), dict(state=None), dict(state_out=None),
    dict(max_blocks_per_seq=0), dict(max_blocks_per_seq=62), dict(n_pages=0), dict(n_slots=-1), dict(slots=None), dict(state_out=PTR),
    dict(lens_out=PTR), dict(lens_out=2 * PTR)])
def test_page_refusals(kw):
    assert _pages(_p(), **kw) == B.ERR_INVALID_ARG


def test_page_sizes():
    assert _pages(_p(t_max=1 << 30, t_stride=1 << 30), max_blocks_per_seq=1 << 26) == B.ERR_UNSUPPORTED     # 3 * 2^30 positions
    assert _pages(_p(batch=0)) == B.ERR_INVALID_ARG
    assert B.lib().ams_assign_pages(C.byref(_p()), None, PTR, PTR, None, None, None, 0, None) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("k,scale", [((2, 3, 4, 100, 64), (2, 3, 4, 7, 4, 16)), ((2, 3, 4, 96, 32), (2, 3, 4, 6, 2, 16))])
def test_scale_shapes(k, scale):
    assert B.scale_shape(torch.empty(k, dtype=torch.uint8)) == scale
    assert B.scale_shape(torch.empty(k, dtype=torch.uint8).view(torch.float4_e2m1fn_x2)) == scale
    assert B.scale_shape(torch.empty((2, 160, 4, 64), dtype=torch.uint8)) == (2, 10, 4, 4, 16)


# ---- the definition ----

def test_codes_are_the_nearest_and_ties_the_even():
    x = np.zeros((1, 32))
    x[0, 0] = 6.0                                       # scale 1
    x[0, 1:15] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, 0.26, 0.74, 2.51, 4.99, -5.01]
    codes, byte = pack_rows(x)
    assert byte.tolist() == [[127]]
    assert values(codes, byte)[0, 1:15].tolist() == [0, 1, 1, 2, 2, 4, 4, 0, -1, 0.5, 0.5, 3, 4, -6]


@pytest.mark.parametrize("largest,byte", [(7.0, 127), (np.nextafter(7.0, 8), 128), (3.5, 126), (3.4, 126), (0.0, 0), (1e-40, 7), (np.inf, 255),
                                          (3.3e38, 253)])
def test_scales_are_the_least_that_take_the_largest_to_seven(largest, byte):
    x = np.zeros((1, 64))
    x[0, 40] = largest
    codes, b = pack_rows(x)
    assert b[0].tolist() == [0, byte]
    if byte == 255:
        assert not codes.any()
    elif largest > 1e-30:                               # off by no more than half of the steps between 4 and 6
        assert abs(values(codes, b)[0, 40] - largest) <= power(byte)


def test_no_code_is_off_by_more_than_half_a_step():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * np.exp(rng.standard_normal((200, 1)))
    codes, byte = pack_rows(x)
    y = values(codes, byte)
    size = np.repeat(power(byte), 32, -1)
    step = np.where(np.abs(x) >= 4 * size, 2, np.where(np.abs(x) >= 2 * size, 1, 0.5)) * size
    assert (np.abs(y - x) <= step / 2 * (1 + 1e-12)).all() and (np.abs(y) <= 6 * size).all()
    assert (LEVELS[codes & 7].reshape(200, 2, 32).max(-1) >= 3.5).all()   # the largest uses the upper half
