"""ams_attend over caches of 4 bits with keys at the end of the range: a code that stands for 2^128 or more is read as infinite.

Where every query is negative in that channel the logit is -inf and the position has probability 0; so it has, exactly, under a key of 2^25, whose
logits lie more than 10^5 below all others.  So the two caches have to give the same bits everywhere: outputs, log-sums, weights."""
import numpy as np
import pytest
import torch

from paper_2605_23200_amd import binding as B
from cache_util import DEV, ROWS, lens_dev, params, same_bits
from micro_util import GROUP, filled

pytestmark = pytest.mark.gpu

CHANNEL = 37


def _queries(shape, dtype, fits_bf16, seed=3):
    q = torch.randn(shape, generator=torch.Generator().manual_seed(seed))
    q[..., CHANNEL] = -q[..., CHANNEL].abs() - 0.5
    if fits_bf16:
        q = q.to(torch.bfloat16)
    return q.to(ROWS[dtype]).to(DEV)


def _set_key(cache, b, h, t, byte, code=7):
    """One channel of a key alone in its 32: 6 * 2^(byte - 127)."""
    codes, scales = cache.get("k", 0, b, h, t)
    part = CHANNEL // GROUP
    codes[part * GROUP:(part + 1) * GROUP] = 0
    codes[CHANNEL], scales[part] = code, byte
    cache.put("k", 0, b, h, t, codes, scales)


def _attend(cache, p, lens, q):
    units = cache.L * cache.B * cache.H
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:4], device=DEV)
    w = torch.zeros((units, p.t_stride), device=DEV)
    ws = torch.full((B.ams_attend_workspace_bytes(p),), 255, dtype=torch.uint8, device=DEV)
    B.ams_attend(p, cache.upload(), lens_dev(lens), q, out, ws, lse, None, w)
    return out, lse, w


def _far_keys(lens, heads, D, group, W, dtype, paged, causal, fits_bf16=True, t_max=200):
    cache = filled((1, len(lens), heads, D), t_max, lens, paged, 4)
    far = cache.copy()
    for b, T in enumerate(lens):
        for h in range(heads):
            for t, byte in ((T - 1, 254), (T // 2, 253), (3, 254)):
                if h == 1 and t == 3:
                    continue                            # (an ordinary key beside the other head's)
                _set_key(cache, b, h, t, 150), _set_key(far, b, h, t, byte)
    p = params((1, len(lens), heads, D), t_max, group=group, window=W, causal=causal, dtype=dtype)
    q = _queries((1, len(lens), heads * group, W, D), dtype, fits_bf16)
    want, got = _attend(cache, p, lens, q), _attend(far, p, lens, q)
    for x, y in zip(got, want):
        assert not torch.isnan(y).any()                 # (a query that sees nothing has lse -inf)
        same_bits(x, y)
    for b, T in enumerate(lens):
        assert (got[2].view(len(lens), heads, -1)[b, :, [T - 1, T // 2]] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,paged", [(1, False), (2, True)])
@pytest.mark.parametrize("group,W", [(1, 17), (2, 24), (3, 40), (1, 32), (5, 51)])
@pytest.mark.parametrize("causal", [False, True])
def test_weights_from_keys_again(D, heads, paged, group, W, causal):
    """More than 16 queries, with and without places for queries that are not there in the last 32: the position's weight is 0."""
    _far_keys([160, 147], heads, D, group, W, "bf16", paged, causal)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,paged", [(1, True), (2, False), (2, True)])
@pytest.mark.parametrize("group,W", [(1, 1), (2, 4), (1, 16), (2, 24), (3, 43)])
@pytest.mark.parametrize("dtype,fits_bf16", [("bf16", True), ("f32", True), ("f32", False)])
def test_logits_and_weights(D, heads, paged, group, W, dtype, fits_bf16):
    """Every kernel and both ways to the weights.  fp32 queries go in as three terms, of which the lower ones may be 0 or have the other sign."""
    _far_keys([160, 147, 9], heads, D, group, W, dtype, paged, W > 1, fits_bf16)


@pytest.mark.parametrize("dtype,fits_bf16", [("bf16", True), ("f32", True), ("f32", False)])
@pytest.mark.parametrize("group,W", [(2, 4), (5, 3), (2, 9)])
def test_in_later_steps(group, W, dtype, fits_bf16):
    """Waves that take several steps, and two heads a wave of up to 16 queries: lengths of up to 40000 allowed."""
    lens, heads, D, t_max = [1900, 1203], 2, 128, 40000
    shape = (1, 2, heads, D)
    cache = filled(shape, 1904, lens, True, 4)
    cache.table = np.concatenate([cache.table, np.full((2, t_max // 16 - cache.table.shape[1]), -1, np.int32)], 1)
    far = cache.copy()
    for b, T in enumerate(lens):
        for i, t in enumerate((T - 1, 600, 601, 33)):
            _set_key(cache, b, i % 2, t, 150), _set_key(far, b, i % 2, t, 253 + i % 2)
    p = params(shape, t_max, group=group, window=W, causal=True, dtype=dtype)
    q = _queries((1, 2, heads * group, W, D), dtype, fits_bf16)
    for x, y in zip(_attend(far, p, lens, q), _attend(cache, p, lens, q)):
        assert torch.isfinite(y).all()
        same_bits(x, y)


@pytest.mark.parametrize("dtype,fits_bf16", [("bf16", True), ("f32", True), ("f32", False)])
@pytest.mark.parametrize("heads,group,W", [(1, 2, 4), (2, 2, 4), (1, 3, 7)])
def test_the_other_sign_and_nothing_but_infinite_keys(heads, group, W, dtype, fits_bf16):
    """A logit of +inf makes the output and the weights of what its queries see no number, and their log-sum not finite; a sequence whose every logit
    is -inf has out 0, lse -inf and no weights."""
    lens, D, T = [100, 20], 64, 100
    cache = filled((1, 2, heads, D), T, lens, False, 4)
    _set_key(cache, 0, 0, 50, 254, 15)                  # -6 * 2^127: +inf for every query
    for t in range(20):
        _set_key(cache, 1, 0, t, 253)
    p = params((1, 2, heads, D), T, group=group, window=W, causal=True, dtype=dtype)
    q = _queries((1, 2, heads * group, W, D), dtype, fits_bf16)
    out, lse, w = _attend(cache, p, lens, q)
    w = w.view(2, heads, T)
    assert torch.isnan(out[0, 0, :group]).all() and not torch.isfinite(lse[0, 0, :group]).any() and torch.isnan(w[0, 0, :T - W + 1]).all()
    assert (out[0, 1, :group] == 0).all() and (lse[0, 1, :group] == -np.inf).all() and (w[1, 0, :20] == 0).all()
    assert torch.isfinite(out[0, :, group:]).all() and torch.isfinite(lse[0, :, group:]).all() and torch.isfinite(w[:, 1:]).all()
