"""ams_attend over pages of 4 bits with 9 to 16 queries a head, where there are positions enough for two heads a wave: what
test_gpu_cache4.py does for up to 8, with its bounds.  (Enough goes by the bound of the lengths, not by the lengths.)"""
import numpy as np
import pytest
import torch

from paper_2605_23200_amd import binding as B
from cache_util import BLOCK, DEV, blocks, lens_dev, params, same_bits
from micro_util import GROUP, filled
from test_gpu_attend4_steps import MicroUnits
from test_gpu_attend_steps import _call, _check, _lens, _steps
from test_gpu_cache import _attend_case

pytestmark = pytest.mark.gpu

D, ENOUGH = 128, 1 << 18


def _wide(cache, t_max):
    """The cache under a longer table: lengths of up to t_max."""
    assert cache.L * cache.B * cache.H * t_max >= ENOUGH and cache.H % 2 == 0
    more = np.full((cache.B, blocks(t_max) - cache.table.shape[1]), -1, np.int32)
    cache.table = np.concatenate([cache.table, more], 1)
    return cache


@pytest.mark.parametrize("heads", [2, 4])
@pytest.mark.parametrize("group,W,causal", [(16, 1, False), (7, 2, True), (3, 3, True), (1, 16, True), (4, 4, False), (1, 9, True), (15, 1, True)])
def test_attend_shapes(group, W, causal, heads):
    """Lengths at the edges of blocks, steps and splits, shorter than the window, empty."""
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 130, 257, 700, 1500]
    _attend_case(_wide(filled((1, len(lens), heads, D), 1504, lens, True, 5), 10007), lens, group, W, "bf16", causal, t_max=10007, t_stride=10010)


@pytest.mark.parametrize("weights,lse", [("same", True), ("zero", False), (None, True), (None, False)])
def test_attend_layers_and_outputs_that_are_left_out(weights, lse):
    _attend_case(_wide(filled((3, 2, 2, D), 300, [300, 77], True, 7), 30000), [300, 77], 3, 4, causal=True, weights=weights, lse=lse, t_max=30000)


def test_attend_one_sequence_over_many_splits():
    _attend_case(filled((1, 1, 2, D), 131072, [9001], True, 6), [9001], 5, 2, causal=True)


@pytest.mark.parametrize("batch,heads,T,group,W,causal", [(48, 4, 4000, 7, 2, True), (64, 4, 2000, 16, 1, False), (33, 2, 5000, 1, 12, True)])
def test_many_steps_a_wave(batch, heads, T, group, W, causal):
    p = params((1, batch, heads, D), T, group=group, window=W, causal=causal, t_stride=T + 3)
    # (_steps is that of a wave that takes one head; with two it takes no fewer: one round of workgroups is one on a CU, not three)
    assert p.units * T >= ENOUGH and _steps(p) >= 3
    cache = MicroUnits(batch, heads, D, T, _lens(batch, T), True, 31)
    q = torch.from_numpy(np.random.default_rng(7).standard_normal((1, batch, heads * group, W, D))).to(torch.bfloat16)
    _check(p, cache, q, causal, "bf16", _call(p, cache, q, given=not causal), [(b, h) for b in range(batch) for h in range(heads) if b < 12 or h == b % heads])


@pytest.mark.parametrize("group,W", [(1, 16), (2, 6)])
def test_no_numbers_and_the_end_of_the_range(group, W):
    """32 channels of a key that are no number make the outputs of the queries that see its position NaN, of a value those 32 outputs; codes
    under scales of 2^126 and 2^127 that are not finite reach the queries that see them alone.  Not other queries, channels, heads; nor
    what lies behind the last position."""
    heads, t_max = 4, 40000
    lens = [160, 147]
    cache = _wide(filled((1, 2, heads, D), 200, lens, True, 4), t_max)
    plain = cache.copy()
    sees = torch.zeros((2, heads, W, D), dtype=torch.bool)
    for b, T in enumerate(lens):
        for h, (name, back, part, byte) in enumerate((("k", 3, 0, 255), ("v", 2, 3, 255), ("v", 5, 0, 253), ("v", 1, 3, 254))):
            codes, scales = cache.get(name, 0, b, h, T - back)
            scales[part], codes[part * GROUP:(part + 1) * GROUP] = byte, 0 if byte == 255 else 7
            cache.put(name, 0, b, h, T - back, codes, scales)
            channel = torch.ones(D, dtype=torch.bool) if name == "k" else torch.arange(D) // GROUP == part
            sees[b, h] = (torch.arange(W) + back >= W)[:, None] & channel
        for h in range(heads):
            for t in range(T, blocks(T) * BLOCK):
                for name in ("k", "v"):
                    cache.put(name, 0, b, h, t, np.full(D, 7), np.full(D // GROUP, 255))
    p = params((1, 2, heads, D), t_max, group=group, window=W, causal=True)
    q = torch.randn((1, 2, heads * group, W, D), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    got = []
    for c in (cache, plain):
        out, w = torch.zeros_like(q), torch.zeros((2 * heads, t_max), device=DEV)
        B.ams_attend(p, c.upload(), lens_dev(lens), q, out, torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV), None, None, w)
        got.append((out.cpu().view(2, heads, group, W, D), w.view(2, heads, t_max)))
    finite = [torch.isfinite(out.float()) for out, _ in got]
    assert finite[1].all()
    for g in range(group):
        assert torch.equal(~finite[0][:, :2, g], sees[:, :2])
        assert not (~finite[0][:, 2:, g] & ~sees[:, 2:]).any()               # (who sees the ends of the range may have a finite sum)
        blind = ~sees.any(-1)                                                # queries that see nothing of it: the same bits
        same_bits(got[0][0][:, :, g][blind], got[1][0][:, :, g][blind])
    same_bits(got[0][1][:, 1], got[1][1][:, 1])                              # (a NaN value changes no weight; see test_gpu_cache4.py for the ends)
    assert torch.isfinite(got[0][1][:, 1:]).all()


def test_two_calls_give_the_same_bits_and_a_graph_replays_them():
    lens = [3000, 1700, 0, 4096]
    cache = MicroUnits(4, 8, D, 10000, lens, True, 9)
    p = params((1, 4, 8, D), 10000, group=7, window=2, causal=True)
    q = torch.randn((1, 4, 56, 2, D), device=DEV).to(torch.bfloat16)
    out, w, at = torch.zeros_like(q), torch.zeros((32, 10000), device=DEV), lens_dev(lens)
    ws, view = torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV), cache.view()
    B.ams_attend(p, view, at, q, out, ws, None, None, w)
    torch.cuda.synchronize()
    first = (out.clone(), w.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ams_attend(p, view, at, q, out, ws, None, None, w)
    for _ in range(3):
        out.zero_(), w.zero_(), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        same_bits(out, first[0])
        for b, n in enumerate(lens):
            same_bits(w.view(4, 8, -1)[b, :, :n].contiguous(), first[1].view(4, 8, -1)[b, :, :n].contiguous())
