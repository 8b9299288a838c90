"""ams_attend over caches of 4 bits where every wave takes several steps of 32 positions, heads two at a time and one at a time: what
test_gpu_attend_steps.py does for 8 bits, with its bounds.  (S there is twice the steps of a wave that takes one head, and two more; with two
heads a split is at most one and a half times as long.)"""
import numpy as np
import pytest
import torch

from paper_2605_23200_amd import binding as B
from cache_util import BLOCK, DEV, ROWS, blocks, params
from micro_util import GROUP, LEVELS
from test_gpu_attend_steps import SHAPES, _call, _check, _lens, _steps

pytestmark = pytest.mark.gpu


class MicroUnits:
    """A cache of one layer whose codes and scale bytes are made as such, per (sequence, head); what lies behind a sequence is no number."""

    def __init__(self, batch, heads, dim, capacity, lens, paged, seed):
        self.shape, self.lens = (1, batch, heads, dim), lens
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
            codes = torch.full(lead + (dim // 2,), 0x77, dtype=torch.uint8, device=DEV)
            scale = torch.full(scales + (dim // GROUP, BLOCK), 255, dtype=torch.uint8, device=DEV)
            for b, n in enumerate(lens):
                if n == 0:
                    continue
                x = rng.integers(0, 256, (heads, n, dim // 2), dtype=np.uint8)
                s = rng.integers(118, 124, (heads, dim // GROUP, n))
                if name == "k":
                    s = s - 2 + self.loudness(heads, n)[:, None]
                self.host[name, b] = (x, s)
                part = torch.from_numpy(x).to(DEV)
                whole = torch.full((heads, dim // GROUP, blocks(n) * BLOCK), 255, dtype=torch.uint8)
                whole[:, :, :n] = torch.from_numpy(s.astype(np.uint8))
                whole = whole.unflatten(-1, (-1, BLOCK)).transpose(1, 2).to(DEV)          # [heads, blocks, groups, 16]
                if table is None:
                    codes[0, b, :, :n], scale[0, b, :, :blocks(n)] = part, whole
                    continue
                page = torch.from_numpy(table[b, :blocks(n)]).long().to(DEV)
                t = torch.arange(n, device=DEV)
                codes[0, page[t // BLOCK] * BLOCK + t % BLOCK] = part.transpose(0, 1)
                scale[0, page] = whole.transpose(0, 1)
            self.dev[name], self.dev[name + "_scale"] = codes, scale
        self.table = torch.from_numpy(table).to(DEV) if paged else None

    @staticmethod
    def loudness(heads, n):
        """Exponents of keys by head: alike, the largest logits early, late, and louder from stretch to stretch (the reference moves again and again)."""
        s = np.zeros((heads, n), dtype=np.int64)
        s[1 % heads, :20] = 3
        s[2 % heads, -20:] = 3
        s[3 % heads] = np.floor(np.linspace(-3, 3.99, n))
        return s

    def view(self):
        d = self.dev
        return B.cache_view(d["k"], d["v"], d["k_scale"], d["v_scale"], block_table=self.table)

    def rows(self, name, b, h):
        if self.lens[b] == 0:
            return np.zeros((0, self.shape[3]))
        x, s = (y[h] for y in self.host[name, b])
        codes = np.stack([x & 15, x >> 4], -1).reshape(len(x), -1).astype(np.int64)
        value = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
        return value * np.repeat(2.0 ** (s.T - 127.0), GROUP, 1)


@pytest.mark.parametrize("batch,heads,T,group,W,causal,least", SHAPES + [(64, 4, 2000, 2, 4, True, 5), (64, 4, 2000, 1, 1, False, 5), (80, 3, 2000, 4, 1, True, 5)])
@pytest.mark.parametrize("dtype,D,paged", [("bf16", 128, True), ("bf16", 64, False), ("f32", 128, False), ("f32", 64, True)])
def test_many_steps_a_wave(batch, heads, T, group, W, causal, least, dtype, D, paged):
    p = params((1, batch, heads, D), T, group=group, window=W, dtype=dtype, causal=causal, t_stride=T + 3)
    assert _steps(p) >= least
    cache = MicroUnits(batch, heads, D, T, _lens(batch, T), paged, 31)
    q = torch.from_numpy(np.random.default_rng(7).standard_normal((1, batch, heads * group, W, D))).to(ROWS[dtype])
    # (of the many short sequences one head each)
    _check(p, cache, q, causal, dtype, _call(p, cache, q, given=not causal), [(b, h) for b in range(batch) for h in range(heads) if b < 21 or h == b % heads])


@pytest.mark.parametrize("heads", [2, 3])
def test_no_number_in_a_later_step(heads):
    """A value that is no number deep inside a split: 32 outputs of the queries that see it, and nothing else of the pair."""
    batch, T, D, W = 96, 2300, 128, 2
    lens = [T - 7 * (b % 40) for b in range(batch)]
    cache = MicroUnits(batch, heads, D, T, lens, True, 5)
    want = torch.zeros((batch, heads, W, D), dtype=torch.bool)
    for b, h, back, part in ((3, 0, 1, 2), (50, 1, 2, 0), (77, heads - 1, 700, 3)):
        t = lens[b] - back
        cache.dev["v_scale"][0, int(cache.table[b, t // BLOCK]), h, part, t % BLOCK] = 255
        want[b, h, :, part * GROUP:(part + 1) * GROUP] = (torch.arange(W) + lens[b] - W >= t)[:, None]
    p = params((1, batch, heads, D), T, group=2, window=W, causal=True)
    q = torch.randn((1, batch, heads * 2, W, D)).to(torch.bfloat16)
    out, _, w, _ = _call(p, cache, q)
    nan = torch.isnan(torch.from_numpy(out))[0].unflatten(1, (heads, 2))
    for g in range(2):
        assert torch.equal(nan[:, :, g], want)
    assert not np.isnan(w[:, :min(lens)]).any()
