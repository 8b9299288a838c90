"""ams_attend where every wave takes several steps of 32 positions (many units, so that a split is long): the running reference that
moves and rescales, names, codes and scales fetched a step or two ahead, the end of a sequence inside a later step, weights kernels
with several steps; against the definition in 64 bits.

Tolerances: those derived in test_gpu_cache.py for one step (err_p of a probability; 2^-16 or 2^-22 for the terms of the second product),
and what the steps S of a wave add, each rounding 2^-24 of the running magnitude: the sum takes 8 additions and one rescaling a step
(10 S), an output at most 8 roundings in each product of the 2 (fp32: 3) terms and one rescaling (18 S, 26 S).  The waves of a workgroup and
the splits are joined with two roundings each, of at most 4 and 2: inside the 8 roundings that err_p has in hand."""
import math

import numpy as np
import pytest
import torch

from paper_2605_23200_amd import binding as B
from cache_util import BLOCK, CODE, DEV, ROWS, blocks, lens_dev, params
from test_gpu_cache import _attend_reference

pytestmark = pytest.mark.gpu


class Units:
    """A cache of one layer whose codes and scales are made as such, per (sequence, head); what lies behind a sequence is no number."""

    def __init__(self, kind, batch, heads, dim, capacity, lens, paged, seed, k_scale=None):
        self.shape, self.lens, self.kind = (1, batch, heads, dim), lens, kind
        rng = np.random.default_rng(seed)
        nb = blocks(capacity)
        if paged:
            counts = [blocks(n) for n in lens]
            order = rng.permutation(sum(counts) + 1)
            table, at = np.full((batch, nb), -1, np.int32), 0
            for b, n in enumerate(counts):
                table[b, :n] = order[at:at + n]
                at += n
            lead, scales = (1, len(order) * BLOCK, heads), (1, len(order), heads)
        else:
            table, lead, scales = None, (1, batch, heads, capacity), (1, batch, heads, nb)
        self.dev, self.host = {}, {}
        for name in ("k", "v"):
            codes = torch.full(lead + (dim,), 127, dtype=torch.uint8, device=DEV)    # e4m3: no number
            scale = torch.full(scales, math.nan, device=DEV)
            for b, n in enumerate(lens):
                if n == 0:
                    continue
                if kind == "int8":
                    x = torch.from_numpy(rng.integers(-127, 128, (heads, n, dim)).astype(np.int8))
                else:
                    x = torch.from_numpy((rng.standard_normal((heads, n, dim)) * 70).clip(-448, 448).astype(np.float32)).to(CODE[kind])
                s = 2.0 ** (rng.integers(-8, -5, (heads, blocks(n))) - 0.0)
                if name == "k" and k_scale:
                    s = k_scale(heads, blocks(n))
                self.put(codes, scale, table, b, x, s)
                self.host[name, b] = (x, s)
            self.dev[name], self.dev[name + "_scale"] = codes.view(CODE[kind]), scale
        self.table = torch.from_numpy(table).to(DEV) if paged else None

    @staticmethod
    def put(codes, scale, table, b, x, s):
        heads, n, dim = x.shape
        s = torch.from_numpy(s.astype(np.float32)).to(DEV)
        x = x.view(torch.uint8).to(DEV)
        if table is None:
            codes[0, b, :, :n], scale[0, b, :, :s.shape[1]] = x, s
            return
        for j in range(s.shape[1]):
            page, part = int(table[b, j]), x[:, j * BLOCK:(j + 1) * BLOCK]
            codes[0, page * BLOCK:page * BLOCK + part.shape[1]] = part.transpose(0, 1)
            scale[0, page] = s[:, j]

    def view(self):
        d = self.dev
        return B.cache_view(d["k"], d["v"], d["k_scale"], d["v_scale"], block_table=self.table)

    def rows(self, name, b, h):
        if self.lens[b] == 0:
            return np.zeros((0, self.shape[3]))
        x, s = self.host[name, b]
        return x[h].to(torch.float32).double().numpy() * np.repeat(s[h], BLOCK)[:x.shape[1], None]


def _splits(p):
    """Splits of the longest sequence, from the workspace that the call asks for (statistics, joined ones, outputs, logits)."""
    up = lambda x: -(-x // 256) * 256
    units, N, D = p.units, p.group * p.window, p.head_dim
    for n in range(1, 4097):
        total = up(units * n * N * 8) + (up(units * n * N * D * 4) if n > 1 else 0)
        total += up(units * blocks(p.t_max) * N * BLOCK * 4) if N <= 16 else up(units * N * 8) if n > 1 else 0
        if total == B.ams_attend_workspace_bytes(p):
            return n
    raise AssertionError("no number of splits fits the workspace")


def _steps(p):
    """Fewest steps that a wave of a whole split takes."""
    N = p.group * p.window
    waves = 4 if N <= 32 else 2 if N <= 64 else 1       # side by side along the positions
    return p.t_max // _splits(p) // (32 * waves)


def _call(p, cache, q, given=True, seed=0):
    units, N = p.units, p.group * p.window
    out, lse = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:4], 9.0, device=DEV)
    w_in = torch.rand((units, p.t_stride), generator=torch.Generator().manual_seed(seed)) * 4
    w_out = torch.full((units, p.t_stride), -5.0, device=DEV)
    ws = torch.full((B.ams_attend_workspace_bytes(p),), 255, dtype=torch.uint8, device=DEV)       # NaN wherever it is read unwritten
    B.ams_attend(p, cache.view(), lens_dev(cache.lens), q.to(DEV), out, ws, lse, w_in.to(DEV) if given else None, w_out)
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), w_out.double().cpu().numpy(), w_in.double().numpy() * given


def _check(p, cache, q, causal, dtype, results, which=None):
    _, Bt, H, D = cache.shape
    group, W = p.group, p.window
    out, lse, w, w_in = results
    hq = q.double().numpy()
    S = 2 * _steps(p) + 2                               # at most: the last split may be a short one
    last, half, a_step = (2.0 ** -16, 2.0 ** -8, 18) if dtype == "bf16" else (2.0 ** -22, 2.0 ** -24, 26)
    for b in range(Bt):
        for h in range(H):
            if which and (b, h) not in which:
                continue
            unit, T = b * H + h, cache.lens[b]
            k, v = cache.rows("k", b, h), cache.rows("v", b, h)
            want, want_lse, pr, A = _attend_reference(hq[0, b, h * group:(h + 1) * group].reshape(group * W, D), k, v, W, causal)
            err_sum = 10 * S * 2.0 ** -24
            err_p = 32 * 2.0 ** -24 * A + 2.0 ** -21 + err_sum
            got = out[0, b, h * group:(h + 1) * group].reshape(group * W, D)
            terms = pr @ np.abs(v) if T else np.zeros_like(want)
            bound = half * np.abs(want) + (2 * err_p[:, None] + last + a_step * S * 2.0 ** -24) * terms + 1e-37
            assert (np.abs(got - want) <= bound).all(), (b, h, T, (np.abs(got - want) / bound).max())
            x = lse[0, b, h * group:(h + 1) * group].reshape(-1)
            empty = ~np.isfinite(want_lse)
            assert (x[empty] == -np.inf).all()
            x, y, e = x[~empty], want_lse[~empty], err_p[~empty]
            assert (np.abs(x - y) <= e + 2.0 ** -22 * np.abs(y)).all(), (b, h, T)
            start, more = w_in[unit, :T], pr.sum(0)
            bound = 2 * (err_p[:, None] * pr).sum(0) + 2.0 ** -22 * more + 2.0 ** -23 * (start + more) + 1e-37
            assert (np.abs(w[unit, :T] - start - more) <= bound).all(), (b, h, T)
            assert (w[unit, T:] == -5).all()


def _loudness(heads, n):
    """Scales of keys by head: alike, the largest logits early, late, and louder from block to block (the reference moves again and again)."""
    s = np.full((heads, n), 2.0 ** -7)
    s[1 % heads, :2] = 2.0 ** -4
    s[2 % heads, -2:] = 2.0 ** -4
    s[3 % heads] = 2.0 ** np.floor(np.linspace(-10, -3.01, n))
    return s


def _lens(batch, T):
    """Ends around steps and splits, whole rows, and short ones for the rest."""
    some = [T, T - 1, T - 15, T - 16, T - 17, T - 31, T - 32, T - 33, T - 100, T // 2, T // 2 + 1, 129, 128, 160, 257, 0, 1, 512, 513, 640, T // 3]
    return (some + [(37 * i) % 300 for i in range(batch)])[:batch]


# batch, heads, t_max; group, window, causal; steps that a wave takes at least
SHAPES = [(64, 4, 2000, 4, 1, False, 5), (64, 4, 2000, 4, 4, True, 5), (64, 4, 4000, 7, 1, True, 3), (64, 4, 2000, 4, 8, False, 7),
          (64, 4, 2000, 3, 7, True, 7), (64, 4, 2000, 8, 5, True, 15), (64, 4, 2000, 8, 16, False, 30), (64, 4, 2000, 8, 16, True, 30)]


@pytest.mark.parametrize("batch,heads,T,group,W,causal,least", SHAPES)
@pytest.mark.parametrize("kind,dtype,D,paged", [("int8", "bf16", 128, True), ("e4m3", "bf16", 64, False), ("e4m3", "f32", 128, False),
                                                ("int8", "f32", 64, True)])
def test_many_steps_a_wave(batch, heads, T, group, W, causal, least, kind, dtype, D, paged):
    p = params((1, batch, heads, D), T, group=group, window=W, dtype=dtype, causal=causal, t_stride=T + 3)
    assert _steps(p) >= least, _steps(p)
    cache = Units(kind, batch, heads, D, T, _lens(batch, T), paged, 31, _loudness)
    q = torch.from_numpy(np.random.default_rng(7).standard_normal((1, batch, heads * group, W, D))).to(ROWS[dtype])
    # (of the many short sequences one head each)
    _check(p, cache, q, causal, dtype, _call(p, cache, q, given=not causal), [(b, h) for b in range(batch) for h in range(heads) if b < 21 or h == b % heads])


def test_many_steps_of_2048_positions_a_workgroup():
    """17 to 32 queries over so many units that a split is of 2048 positions: sixteen steps a wave, ends in the first, a middle and the last."""
    batch, heads, T = 64, 8, 6200
    p = params((1, batch, heads, 64), T, group=4, window=5, causal=True, t_stride=T)
    assert _splits(p) == 4 and _steps(p) >= 12
    lens = [T, T - 1, 6145, 6144, 4097, 4095, 2048, 2049, 2017, 1000] + [(53 * i) % 200 for i in range(batch - 10)]
    cache = Units("e4m3", batch, heads, 64, T, lens, True, 33, _loudness)
    q = torch.from_numpy(np.random.default_rng(8).standard_normal((1, batch, heads * 4, 5, 64))).to(torch.bfloat16)
    _check(p, cache, q, True, "bf16", _call(p, cache, q), [(b, h) for b in range(batch) for h in range(heads) if b < 10 or h == b % heads])


@pytest.mark.parametrize("group,W", [(1, 1), (2, 10), (5, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_probabilities_with_large_values_in_consecutive_steps(group, W, dtype):
    """A position of probability 2^-40 whose values are 2^60 carries the output: in the step of a wave after the one that sets the
    reference, in the one before it (what was summed is scaled down by 2^-40 and not lost), and two steps away."""
    batch, T, D = 256, 2000, 64
    p = params((1, batch, 1, D), T, group=group, window=W, dtype=dtype)
    waves = 4 if group * W <= 32 else 2
    assert _steps(p) >= 4
    n = 5 * 32 * waves + 7
    cache = Units("int8", batch, 1, D, T, [n] * 4 + [40] * (batch - 4), False, 35)
    step = 32 * waves
    for b, (loud, small) in enumerate(((0, step + 8), (step, 8), (2 * step, 3), (5, 3 * step + 17))):
        k, ks = torch.zeros((1, n, D), dtype=torch.int8), np.ones((1, blocks(n)))
        v, vs = torch.ones((1, n, D), dtype=torch.int8), np.ones((1, blocks(n)))
        k[0, loud:loud + 8, 0], k[0, small, 0] = 127, 127 - 28
        j = small // BLOCK
        v[0, j * BLOCK:(j + 1) * BLOCK] = 0
        v[0, small], vs[0, j] = 64, 2.0 ** 54
        for name, x, s in (("k", k, ks), ("v", v, vs)):
            cache.host[name, b] = (x, s)
            Units.put(cache.dev[name].view(torch.uint8), cache.dev[name + "_scale"], None, b, x, s)
    q = torch.zeros((1, batch, group, W, D), dtype=ROWS[dtype])
    q[..., 0] = 8.0                                     # logits of 127 and 99
    results = _call(p, cache, q)
    assert results[0][0, :4].min() > 1e4
    _check(p, cache, q, False, dtype, results, [(b, 0) for b in range(4)])


@pytest.mark.parametrize("group,W", [(1, 16), (1, 24), (2, 24)])
def test_no_numbers_in_a_later_step(group, W):
    """A block of K, of V, or a query that is no number, several steps into a split: what sees it and nothing else."""
    batch, heads, T, D = 64, 4, 2000, 64
    p = params((1, batch, heads, D), T, group=group, window=W, causal=True)
    assert _steps(p) >= 5
    n = 632                                             # the first queries of the window see nothing of the last block
    lens = [n, n, n, 1500] + [33] * (batch - 4)
    cache = Units("int8", batch, heads, D, T, lens, False, 37, _loudness)
    first = n // BLOCK * BLOCK
    cache.dev["k_scale"][0, 0, 1, n // BLOCK] = math.nan
    cache.dev["v_scale"][0, 1, 2, n // BLOCK] = math.nan
    cache.dev["v_scale"][0, 3, 0, 20] = math.nan        # in the middle: every query sees it
    q = torch.from_numpy(np.random.default_rng(9).standard_normal((1, batch, heads * group, W, D))).to(torch.bfloat16)
    q[0, 2, 0, 0] = math.nan                            # the first query of head 0's window: sees n - W + 1 positions
    results = _call(p, cache, q)
    out, w = results[0][0], results[2].reshape(batch, heads, T)
    sees = n - W + np.arange(W) >= first
    assert sees.any() and not sees.all()
    nan_out, nan_w = np.zeros(out.shape, bool), np.zeros(w.shape, bool)
    nan_out[0, group:2 * group, sees] = True
    nan_w[0, 1, :n] = True                              # the last query's sum is no number, and it sees all
    nan_out[1, 2 * group:3 * group, sees] = True        # (values that are no number leave the weights alone)
    nan_out[3, :group] = True
    nan_out[2, 0, 0] = True
    nan_w[2, 0, :n - W + 1] = True
    assert (np.isnan(out) == nan_out).all() and (np.isnan(w) == nan_w).all()
    bad = {(0, 1), (1, 2), (3, 0), (2, 0)}
    _check(p, cache, q, True, "bf16", results, [(b, h) for b in range(6) for h in range(heads) if (b, h) not in bad])
