"""Refusals of the entry points around a bounded cache, on the host: statuses before anything is launched, and the binding's checks.
The table of rotary frequencies against its formulas."""
import ctypes as C
import math

import pytest
import torch

from paper_2605_23200_amd import binding as B

PTR = 4096                                             # never followed: every call here ends at its checks


def _p(**kw):
    d = dict(n_layers=2, batch=3, n_kv_heads=4, group=2, window=8, t_max=1000, budget=200, n_segments=1)
    d.update(kw)
    return B.make_params(**d)


def _dense(dtype=B.INT8, base=PTR, cap=1000, k_scale=PTR, v_scale=PTR):
    return B.Cache(B.KvView(B.LAYOUT_DENSE, base, base + 16 if base else None, cap, None, 0, 0, 0), dtype, k_scale, v_scale)


def _paged(dtype=B.INT8, table=PTR, max_blocks=63, block=16, slots=160000):
    return B.Cache(B.KvView(B.LAYOUT_PAGED, PTR, PTR, 0, table, max_blocks, block, slots), dtype, PTR, PTR)


def _attend(p, c, lens=PTR, q=PTR, out=2 * PTR, lse=None, win=None, wout=None, ws=PTR, n=1 << 40):
    return B.lib().ams_attend(C.byref(p), C.byref(c) if c is not None else None, lens, q, out, lse, win, wout, ws, n, None)


def _recode(p, src, dst, lens=PTR, idx=None, n_kept=None):
    return B.lib().ams_recode(C.byref(p), C.byref(src), lens, idx, n_kept, C.byref(dst), None, None, None)


def _evict(p, src, dst, lens=PTR, w=PTR, wout=2 * PTR, idx=PTR, n_kept=PTR, lens_out=None, ws=PTR, n=1 << 40):
    return B.lib().ams_evict(C.byref(p), C.byref(src), lens, w, C.byref(dst), wout, idx, n_kept, lens_out, ws, n, None)


def _tokens(**kw):
    d = dict(q=PTR, k=PTR, v=PTR, q_stride=2 * 4 * 128, k_stride=4 * 128, v_stride=4 * 128, q_weight=None, k_weight=None, norm_eps=1e-6,
             positions=None, n_new=1)
    d.update(kw)
    return B.NewTokens(*d.values())


def _append(p, c, x, rope=None, lens=PTR, q_out=1 << 20, lens_out=None):
    return B.lib().ams_append(C.byref(p), C.byref(x), C.byref(rope) if rope is not None else None, lens, q_out, C.byref(c), lens_out, None)


BAD_SIZES = [("n_layers", 0, B.ERR_INVALID_ARG), ("batch", 0, B.ERR_INVALID_ARG), ("group", 0, B.ERR_INVALID_ARG),
             ("t_max", 0, B.ERR_INVALID_ARG), ("t_stride", 999, B.ERR_INVALID_ARG), ("kv_dtype", B.INT8, B.ERR_INVALID_ARG),
             ("head_dim", 96, B.ERR_UNSUPPORTED), ("n_layers", 10000, B.ERR_UNSUPPORTED), ("t_max", 1 << 31 - 1, B.ERR_INVALID_ARG)]


@pytest.mark.parametrize("field,value,status", BAD_SIZES)
def test_bad_sizes(field, value, status):
    p = _p()
    setattr(p, field, value)
    assert _attend(p, _dense()) == status and _recode(p, _dense(), _dense(base=1 << 20)) == status
    assert _evict(p, _dense(), _dense(base=1 << 20)) == status and _append(p, _dense(), _tokens()) == status
    assert B.ams_attend_workspace_bytes(p) == 0 and B.ams_evict_workspace_bytes(p) == 0


@pytest.mark.parametrize("t_max", [(1 << 30) + 1, (1 << 31) - 1])
def test_lengths_beyond_the_kernels_positions(t_max):
    """Positions are 32-bit numbers with room above them: longer caches are refused whatever the rows and strides hold."""
    p = _p(t_max=t_max, t_stride=t_max, budget=200)
    src, dst = _dense(cap=t_max), _dense(base=1 << 20, cap=t_max)
    assert _attend(p, src) == B.ERR_UNSUPPORTED and _append(p, src, _tokens()) == B.ERR_UNSUPPORTED
    assert _recode(p, src, dst) == B.ERR_UNSUPPORTED and _evict(p, src, dst) == B.ERR_UNSUPPORTED
    assert B.ams_attend_workspace_bytes(p) == 0 and B.ams_evict_workspace_bytes(p) == 0
    p = _p(t_max=1 << 30, t_stride=1 << 30)             # the longest
    assert B.ams_attend_workspace_bytes(p) > 0 and B.ams_evict_workspace_bytes(p) > 0
    assert _attend(p, _dense(cap=1 << 30), n=0) == B.ERR_WORKSPACE_TOO_SMALL


def test_a_stride_shorter_than_the_row():
    p = _p(t_max=1000, t_stride=999)
    assert _attend(p, _dense()) == B.ERR_INVALID_ARG and _evict(p, _dense(), _dense(base=1 << 20)) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("cache,status", [
    (_dense(base=None), B.ERR_INVALID_ARG), (_dense(base=PTR + 8), B.ERR_INVALID_ARG), (_dense(cap=999), B.ERR_INVALID_ARG),
    (_dense(k_scale=None), B.ERR_INVALID_ARG), (_dense(v_scale=None), B.ERR_INVALID_ARG), (_dense(dtype=9), B.ERR_INVALID_ARG),
    (_dense(dtype=B.F32), B.ERR_INVALID_ARG),          # rows of another type than the parameters'
    (_paged(table=None), B.ERR_INVALID_ARG), (_paged(max_blocks=62), B.ERR_INVALID_ARG), (_paged(block=32), B.ERR_UNSUPPORTED),
    (_paged(slots=8), B.ERR_INVALID_ARG), (_paged(slots=160008), B.ERR_INVALID_ARG)])
def test_bad_caches(cache, status):
    assert _attend(_p(), cache) == status
    assert _append(_p(), cache, _tokens()) == status
    assert _recode(_p(), cache, _dense(base=1 << 20)) == status and _recode(_p(), _dense(base=1 << 20), cache) == status
    assert _evict(_p(), cache, _dense(base=1 << 20)) == status


def test_attend_refusals():
    p = _p()
    need = B.ams_attend_workspace_bytes(p)
    assert need > 0
    assert _attend(p, _dense(), n=need - 1) == B.ERR_WORKSPACE_TOO_SMALL
    assert _attend(p, None) == B.ERR_INVALID_ARG
    for kw in (dict(lens=None), dict(q=None), dict(out=None), dict(ws=None), dict(win=PTR), dict(q=PTR + 2), dict(out=PTR)):
        assert _attend(p, _dense(), **kw) == B.ERR_INVALID_ARG, kw
    assert _attend(p, _dense(dtype=B.BF16)) == B.ERR_UNSUPPORTED        # rows of kv_dtype
    q = _p(window=129)
    assert _attend(q, _dense()) == B.ERR_UNSUPPORTED and B.ams_attend_workspace_bytes(q) == 0
    q = _p()
    q.causal = 3
    assert _attend(q, _dense()) == B.ERR_INVALID_ARG


def test_recode_refusals():
    p = _p()
    assert _recode(p, _dense(), _dense()) == B.ERR_INVALID_ARG          # in place
    assert _recode(p, _dense(dtype=B.BF16), _dense(dtype=B.BF16, base=1 << 20)) == B.ERR_UNSUPPORTED
    assert _recode(p, _dense(), _dense(base=1 << 20), lens=None) == B.ERR_INVALID_ARG
    assert _recode(p, _dense(), _dense(base=1 << 20), idx=PTR) == B.ERR_INVALID_ARG
    assert _recode(p, _dense(), _dense(base=1 << 20, cap=199), idx=PTR, n_kept=PTR) == B.ERR_INVALID_ARG


def test_evict_refusals():
    p = _p()
    src, dst = _dense(), _dense(base=1 << 20)
    for kw in (dict(lens=None), dict(w=None), dict(wout=None), dict(wout=PTR), dict(idx=None), dict(n_kept=None), dict(ws=None),
               dict(ws=PTR + 8), dict(lens_out=PTR)):
        assert _evict(p, src, dst, **kw) == B.ERR_INVALID_ARG, kw
    assert _evict(p, src, src) == B.ERR_INVALID_ARG
    assert _evict(p, src, dst, n=B.ams_evict_workspace_bytes(p) - 1) == B.ERR_WORKSPACE_TOO_SMALL
    for field, value in (("budget", 0), ("n_sink", -1), ("n_last", -1)):
        q = _p()
        setattr(q, field, value)
        assert _evict(q, src, dst) == B.ERR_INVALID_ARG and B.ams_evict_workspace_bytes(q) == 0


def test_evict_budget_beyond_its_counters():
    """The tail of a row of idx is written by a 32-bit counter in steps of a workgroup: a budget near 2^31 would carry it past its end."""
    p = _p()
    p.budget = (1 << 30) + 1
    assert _evict(p, _dense(), _dense(base=1 << 20)) == B.ERR_UNSUPPORTED and B.ams_evict_workspace_bytes(p) == 0
    p.budget = 1 << 30
    assert B.ams_evict_workspace_bytes(p) > 0


def test_append_refusals():
    p, c = _p(), _dense()
    for kw in (dict(k=None), dict(v=None), dict(q=None), dict(n_new=0), dict(norm_eps=-1.0), dict(norm_eps=math.inf), dict(norm_eps=math.nan),
               dict(q=PTR + 2), dict(k=PTR + 8), dict(v=PTR + 4), dict(q_weight=PTR + 2), dict(k_weight=PTR + 2), dict(q_stride=1023),
               dict(k_stride=511), dict(v_stride=500), dict(k_stride=516), dict(q_stride=1028)):
        assert _append(p, c, _tokens(**kw)) == B.ERR_INVALID_ARG, kw
    assert _append(p, c, _tokens(), q_out=None) == B.ERR_INVALID_ARG
    assert _append(p, c, _tokens(q=2 * PTR), q_out=2 * PTR) == B.ERR_INVALID_ARG       # in place
    assert _append(p, c, _tokens(), lens=None) == B.ERR_INVALID_ARG
    assert _append(p, c, _tokens(), lens_out=PTR) == B.ERR_INVALID_ARG
    assert _append(p, c, _tokens(n_new=(1 << 20) + 1)) == B.ERR_UNSUPPORTED
    for field, value in (("layout", 2), ("rot_dim", 130), ("rot_dim", 3), ("rot_dim", -2), ("gain", math.inf)):
        r = B.make_rope(128)
        setattr(r, field, value)
        assert _append(p, c, _tokens(), rope=r) == B.ERR_INVALID_ARG, field
    r = B.make_rope(128)
    r.freq[3] = math.nan
    assert _append(p, c, _tokens(), rope=r) == B.ERR_INVALID_ARG
    small = _p(head_dim=64)
    x = _tokens(q_stride=512, k_stride=256, v_stride=256)
    assert _append(small, c, x, rope=B.make_rope(128)) == B.ERR_INVALID_ARG    # rotates more channels than there are


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=130), dict(rot_dim=-2), dict(layout=2), dict(scaling=4), dict(base=0.0),
                                dict(base=math.inf), dict(gain=math.nan), dict(scaling=B.ROPE_LINEAR, factor=0.5),
                                dict(scaling=B.ROPE_BASE, factor=2.0, rot_dim=2), dict(scaling=B.ROPE_BY_PARTS, factor=2.0),
                                dict(scaling=B.ROPE_BY_PARTS, factor=2.0, original_len=100, slow=4.0, fast=4.0)])
def test_rope_refusals(kw):
    with pytest.raises(B.AmsError) as e:
        B.make_rope(**dict(dict(rot_dim=64), **kw))
    assert e.value.status == B.ERR_INVALID_ARG
    assert B.lib().ams_rope_init(None, 0, 64, 1e4, 0, 1.0, 0, 1.0, 32.0, 1.0) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("n", [0, 2, 6, 64, 128])
@pytest.mark.parametrize("scaling", [B.ROPE_PLAIN, B.ROPE_LINEAR, B.ROPE_BASE, B.ROPE_BY_PARTS])
def test_rope_frequencies(n, scaling):
    if scaling == B.ROPE_BASE and n == 2:
        return
    r = B.make_rope(n, base=5e5, scaling=scaling, factor=8.0, original_len=8192, slow=1.0, fast=4.0, gain=1.25)
    assert r.rot_dim == n and r.gain == 1.25 and all(r.freq[i] == 0 for i in range(n // 2, 64))
    for i in range(n // 2):
        base = 5e5 * 8.0 ** (n / (n - 2)) if scaling == B.ROPE_BASE else 5e5
        f = math.exp(-2 * i / n * math.log(base))
        if scaling == B.ROPE_LINEAR:
            f /= 8
        if scaling == B.ROPE_BY_PARTS:
            turns = 8192 * f / (2 * math.pi)
            c = min(1.0, max(0.0, (turns - 1) / 3))
            f = f * c + f / 8 * (1 - c)
        assert r.freq[i] == pytest.approx(f, rel=1e-13)
    if scaling == B.ROPE_BY_PARTS and n == 128:        # both ends and the ramp are there
        plain = B.make_rope(n, base=5e5)
        kinds = {round(plain.freq[i] / r.freq[i], 6) for i in range(64)}
        assert 1.0 in kinds and 8.0 in kinds and len(kinds) > 2


def test_binding_checks():
    k = torch.zeros((1, 1, 2, 32, 64), dtype=torch.int8)
    with pytest.raises(ValueError):
        B.cache_view(k, k)                             # not on a GPU
    assert B.scale_shape(k) == (1, 1, 2, 2)
    assert B.scale_shape(torch.zeros((3, 48, 2, 64))) == (3, 3, 2)
    assert B.scale_shape(torch.zeros((1, 1, 2, 33, 64))) == (1, 1, 2, 3)


def test_workspace_grows_with_the_work():
    small, large = B.ams_attend_workspace_bytes(_p()), B.ams_attend_workspace_bytes(_p(batch=6))
    assert 0 < small < large
