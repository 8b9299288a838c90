"""ams_attend over caches of 4 bits, two heads a wave: how many positions a workgroup takes, the workspace that this needs, and the definition in 64
bits where a wave takes many steps, with the steps that it really takes.

Tolerances: those of test_gpu_attend_steps.py, whose S is the steps of a wave.  For pairs of heads S follows from their own stretches (_chunk): a step
adds 8 probabilities to a sum and 8 rows in each of the 2 (fp32: 3) products to an output, as with one head a wave (the other head's lanes add zeros,
which round nothing)."""
import numpy as np
import pytest
import torch

import test_gpu_attend_steps
from cache_util import ROWS, blocks, params
from micro_util import filled
from test_gpu_attend4_steps import MicroUnits
from test_gpu_attend_steps import _call, _check, _lens
from test_gpu_cache import _attend_case

pytestmark = pytest.mark.gpu

STEP = 128                                              # positions of the four waves of a workgroup


def _up(a, b):
    return -(-a // b)


def _chunk(units, t_max, three_terms_of_128, pairs):
    """Positions a workgroup takes of up to 16 queries: 512 where that gives 2048 workgroups; else one round of workgroups (pairs: one on a CU; one
    head: three, or two), or, for pairs that would leave a quarter of the CUs empty, 512 again in no more splits than one head takes."""
    work = units // 2 if pairs else units
    if work * _up(t_max, 512) >= 2048:
        return 512
    splits = max(1, 256 * (1 if pairs else 2 if three_terms_of_128 else 3) // work)
    if pairs and 4 * splits * work <= 3 * 256:
        most = _up(t_max, _chunk(units, t_max, three_terms_of_128, False))
        return max(512, _up(_up(t_max, most), STEP) * STEP)
    return _up(_up(t_max, splits), STEP) * STEP


# batch, heads, t_max; group, window, causal; positions a workgroup takes
@pytest.mark.parametrize("batch,heads,T,group,W,causal,chunk", [
    (64, 4, 4000, 7, 1, True, 2048), (64, 4, 2000, 4, 2, False, 1024), (32, 4, 6000, 3, 2, True, 1536), (66, 4, 4000, 4, 1, True, 512),
    (66, 4, 2177, 2, 4, True, 1152), (44, 4, 2500, 8, 1, False, 640), (96, 4, 3000, 1, 3, True, 512)])
@pytest.mark.parametrize("dtype,D,paged", [("bf16", 128, True), ("bf16", 64, False), ("f32", 64, True)])
def test_many_steps(batch, heads, T, group, W, causal, chunk, dtype, D, paged, monkeypatch):
    _steps_case(batch, heads, T, group, W, causal, chunk, dtype, D, paged, monkeypatch)


@pytest.mark.parametrize("batch,heads,T,group,W,causal,chunk", [(64, 4, 4000, 7, 2, True, 2048), (66, 4, 4000, 16, 1, False, 512), (32, 4, 6000, 1, 12, True, 1536)])
def test_many_steps_of_more_queries(batch, heads, T, group, W, causal, chunk, monkeypatch):
    _steps_case(batch, heads, T, group, W, causal, chunk, "bf16", 128, True, monkeypatch)


def _steps_case(batch, heads, T, group, W, causal, chunk, dtype, D, paged, monkeypatch):
    assert _chunk(batch * heads, T, dtype == "f32" and D == 128, True) == chunk
    S = chunk // STEP
    monkeypatch.setattr(test_gpu_attend_steps, "_steps", lambda p: (S - 1) // 2)    # _check doubles it and adds two: S or S + 1
    p = params((1, batch, heads, D), T, group=group, window=W, dtype=dtype, causal=causal, t_stride=T + 3)
    cache = MicroUnits(batch, heads, D, T, _lens(batch, T), paged, 31)
    q = torch.from_numpy(np.random.default_rng(7).standard_normal((1, batch, heads * group, W, D))).to(ROWS[dtype])
    _check(p, cache, q, causal, dtype, _call(p, cache, q, given=not causal), [(b, h) for b in range(batch) for h in range(heads) if b < 21 and h == b % heads])


@pytest.mark.parametrize("seed", range(12))
def test_the_workspace_is_enough_for_any_batch(seed):
    """Bounds of the lengths from one block to beyond the sequences, batches on both sides of every round of workgroups: what the query says is what
    the call takes (exactly that much is given), and the results are right."""
    rng = np.random.default_rng(seed)
    for _ in range(3):
        heads = int(rng.choice([2, 4]))
        batch = int(rng.choice([1, 3, 16, 17, 22, 32, 33, 40, 48, 65])) * 4 // heads
        t_max = int(2 ** rng.uniform(8, 15))
        lens = [min(int(n), t_max) for n in rng.integers(0, 40, batch)]
        lens[-1] = min(300, t_max)
        cache = filled((1, batch, heads, 64), 300, lens, True, seed)
        table = np.full((batch, max(blocks(t_max), cache.table.shape[1])), -1, np.int32)
        table[:, :cache.table.shape[1]] = cache.table
        cache.table = table
        _attend_case(cache, lens, int(rng.choice([1, 4, 8])), 1, "f32" if rng.random() < 0.3 else "bf16", True, t_max=t_max)
