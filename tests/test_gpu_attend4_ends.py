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
        assert torch.isfinite(y).all()
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
