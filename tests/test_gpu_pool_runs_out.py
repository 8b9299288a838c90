"""A serving loop over a pool that runs out: sequences that find no page wait, the others go on, and what waits goes on when pages come back.  The
same loop over slabs, which leaves out the same sequences, gives the same bits."""
import pytest
import torch

from paper_2605_23200_amd import binding as B
from cache_util import BLOCK, DEV, blocks, params, same_bits
from test_gpu_cache4 import _Loop

pytestmark = pytest.mark.gpu


class _Waiting(_Loop):
    def __init__(self, batch, pool, free=0):
        super().__init__(batch, pool)
        self.state[0] = torch.tensor([3, free], dtype=torch.int32, device=DEV)

    def step(self, x, got=None):
        """The new tokens of the sequences that find room (got, their lengths then; by ams_assign_pages where there is a pool)."""
        new, HQ = x.shape[2], self.H * self.G
        if self.pool:
            got = self.assign(self.tables[0], self.lens + new, torch.zeros(self.B * new, dtype=torch.int64, device=DEV))
        served = got > self.lens
        at, seen = torch.where(served, self.lens, self.CAP), torch.where(served, got, 0)   # a full sequence takes nothing, an empty one gives 0
        q = torch.empty((self.L, self.B, HQ, new, self.D), dtype=torch.bfloat16, device=DEV)
        B.ams_append(self.p, x[..., :HQ, :], x[..., HQ:HQ + self.H, :], x[..., HQ + self.H:, :], None, None, 0.0, self.rope, self.lens, at, q,
                     self.views[0])
        self.lens = got
        p = params((self.L, self.B, self.H, self.D), self.CAP, group=self.G, window=new, causal=True)
        out, ws = torch.empty_like(q), torch.empty(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)
        B.ams_attend(p, self.views[0], seen, q, out, ws, None, self.weights[0], self.weights[0])
        return out, got


def test_waiting_sequences_lose_nothing():
    batch, free = 5, 14                                 # two pages each for the prompts, four more
    paged, dense = _Waiting(batch, True, free), _Waiting(batch, False)
    before, waits = torch.zeros(batch, dtype=torch.int32, device=DEV), []
    for t in range(60):
        new = 30 if t == 0 else 1
        x = paged.r(paged.L, batch, new, (paged.G + 2) * paged.H, paged.D)
        (a, got), (b, _) = paged.step(x), dense.step(x, paged.lens)
        same_bits(a, b)
        same_bits(paged.weights[0], dense.weights[0])
        assert (a[:, got == before] == 0).all()
        waits.append((got == before).tolist())
        before = got
        if t == 30:
            done = torch.tensor([True, False, True, False, False], device=DEV)
            paged.end(done), dense.end(done)
            before = paged.lens
    assert waits[2] == [False] * 5 and waits[3] == [False] * 4 + [True]      # 33 positions: four pages for five
    assert waits[30] == [True] * 5                                            # 49: none is left
    assert waits[31][4] is False and waits[31][1] is False                    # two sequences ended
    assert paged.lens.tolist()[4] < paged.lens.tolist()[1]
    head, count = paged.state[0].tolist()
    left = [int(paged.ring[(head + i) % paged.n_pages]) for i in range(count)]
    used = [int(v) for b, n in enumerate(paged.lens.tolist()) for v in paged.tables[0][b, :blocks(n)]]
    assert len(set(left + used)) == len(left + used) == free
