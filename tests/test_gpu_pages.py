"""ams_assign_pages against a plain allocator: every output is a whole number and has to be equal."""
import numpy as np
import pytest
import torch

from paper_2605_23200_amd import binding as B
from cache_util import BLOCK, DEV, blocks

pytestmark = pytest.mark.gpu


def _plain(had, want, t_max, table, ring, state, n_slots):
    """The definition, sequence by sequence, with lists."""
    n, width = len(ring), table.shape[1]
    had, want = np.clip(had, 0, t_max), np.clip(want, 0, t_max)
    head, count = state
    ring, out = ring.copy(), np.full(table.shape, -1, np.int64)
    slots, starts, lens = np.full(n_slots, -1, np.int64), [0], []
    taken = asked = given = 0
    for b in range(len(had)):
        p0, p1 = blocks(int(had[b])), blocks(int(want[b]))
        need = max(p1 - p0, 0)
        asked += need
        served = need == 0 or asked <= count
        pages = list(table[b, :p0])
        if served and p1 > p0:
            pages += [ring[(head + taken + i) % n] for i in range(need)]
            taken += need
        if p1 < p0:
            for page in pages[p1:]:
                ring[(head + count + given) % n] = page
                given += 1
            pages = pages[:p1]
        out[b, :len(pages)] = pages
        lens.append(int(want[b]) if served else int(had[b]))
        for i, pos in enumerate(range(int(had[b]), int(want[b]))):
            if served and starts[-1] + i < n_slots:
                slots[starts[-1] + i] = pages[pos // BLOCK] * BLOCK + pos % BLOCK
        starts.append(starts[-1] + max(int(want[b]) - int(had[b]), 0))
    return out, ring, [(head + taken) % n, count - taken + given], slots, starts, lens


def _case(had, want, t_max, room, n_slots=None, width=None, seed=0, in_place=False, spare=7, head=None, extra=True):
    had, want = np.array(had), np.array(want)
    rng = np.random.default_rng(seed)
    batch, width = len(had), width or blocks(t_max)
    used = [blocks(int(n)) for n in np.clip(had, 0, t_max)]
    names = rng.permutation(sum(used) + room + spare)
    table = rng.integers(-50, 1 << 30, (batch, width))     # entries behind a sequence's pages are not read
    at = 0
    for b in range(batch):
        table[b, :used[b]] = names[at:at + used[b]]
        at += used[b]
    n_pages = sum(used) + room + spare
    head = n_pages - room // 2 - 1 if head is None else head
    ring = np.full(n_pages, -77)
    ring[(head + np.arange(room)) % n_pages] = names[at:at + room]
    total = int(np.clip(np.clip(want, 0, t_max) - np.clip(had, 0, t_max), 0, None).sum())
    n_slots = total + 5 if n_slots is None else n_slots
    expect = _plain(had, want, t_max, table, ring, [head, room], n_slots)
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    p = B.make_params(n_layers=1, batch=batch, n_kv_heads=1, group=1, window=1, t_max=t_max, budget=1, n_segments=1)
    t, r, s = i32(table), i32(ring), i32([head, room])
    out = t if in_place else torch.full_like(t, 99)
    s_out, starts, lens = i32([5, 5]), i32([-3] * (batch + 1)), i32([-3] * batch)
    slots = torch.full((n_slots,), -9, dtype=torch.int64, device=DEV)
    B.ams_assign_pages(p, i32(had), i32(want), t, out, r, s, s_out, starts if extra else None, slots, lens if extra else None)
    assert torch.equal(out.cpu().long(), torch.from_numpy(expect[0])), "table"
    assert r.tolist() == expect[1].tolist() and s_out.tolist() == expect[2]
    assert slots.tolist() == expect[3].tolist()
    if extra:
        assert starts.tolist() == expect[4] and lens.tolist() == expect[5]
    if not in_place:
        assert torch.equal(t, i32(table))
    return out


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("had,want", [([0], [0]), ([0], [1]), ([16], [17]), ([15], [16]), ([33], [0]), ([33], [32]), ([0, 0, 0], [64, 1, 17]),
                                      ([5, 40, 64, 0, 31, 32], [6, 41, 10, 64, 0, 33])])
def test_small_batches(had, want, in_place):
    _case(had, want, 64, 20, in_place=in_place)


@pytest.mark.parametrize("room", [0, 1, 2, 3, 4, 5, 6, 100])
def test_sequences_are_served_in_order_as_far_as_the_pages_go(room):
    """Those that ask for none are always served; behind one that finds no room none that asks is, even if it asks for less."""
    _case([10, 16, 0, 30, 16, 48, 0], [11, 40, 20, 31, 17, 16, 3], 64, room)


@pytest.mark.parametrize("n_slots", [0, 1, 40, 300])
def test_fewer_and_more_slots_than_tokens(n_slots):
    _case([0, 20, 3], [50, 21, 3], 64, 30, n_slots=n_slots)


def test_lengths_outside_are_clamped_and_wide_tables():
    _case([-5, 100, 20, 3], [70, -1, 1000, 1 << 30], 64, 30, width=9)
    _case([0, 64], [64, 1], 64, 30, width=1000, extra=False)


@pytest.mark.parametrize("head", [0, 1, 5])
def test_the_ring_goes_round(head):
    _case([0, 64, 16], [64, 0, 64], 64, 8, spare=0, head=head)


@pytest.mark.parametrize("batch,t_max", [(64, 3000), (255, 700), (256, 700), (257, 700), (1000, 300), (2048, 64), (2049, 64), (5000, 40)])
@pytest.mark.parametrize("in_place", [False, True])
def test_large_batches(batch, t_max, in_place):
    rng = np.random.default_rng(batch)
    had = rng.integers(0, t_max + 1, batch)
    want = np.where(rng.random(batch) < 0.3, 0, np.where(rng.random(batch) < 0.5, np.minimum(had + 1, t_max), rng.integers(0, t_max + 1, batch)))
    asked = int(np.clip((want + 15) // 16 - (had + 15) // 16, 0, None).sum())
    _case(had, want, t_max, int(asked * (0.8 if in_place else 1.1)), in_place=in_place, width=blocks(t_max) + 3)


def test_one_long_sequence():
    _case([100], [100000], 100000, 6300, width=7000)


def test_refusals_of_the_binding():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    p = B.make_params(n_layers=1, batch=2, n_kv_heads=1, group=1, window=1, t_max=64, budget=1, n_segments=1)
    good = dict(p=p, lens_from=i32(2), lens_to=i32(2), table=i32(2, 4), table_out=i32(2, 4), ring=i32(9), state=i32(2), state_out=i32(2),
                starts=i32(3), slots=torch.zeros(4, dtype=torch.int64, device=DEV), lens_out=i32(2))
    B.ams_assign_pages(**good)
    for bad in (dict(lens_from=i32(1)), dict(lens_to=i32(2).long()), dict(table=i32(3, 4)), dict(table_out=i32(2, 5)), dict(table=i32(2, 4).cpu()),
                dict(ring=i32(3, 3)), dict(ring=i32(9)[::2]), dict(state=i32(1)), dict(starts=i32(2)), dict(slots=i32(4)), dict(lens_out=i32(1)),
                dict(table=i32(4, 2).t())):
        with pytest.raises(ValueError):
            B.ams_assign_pages(**dict(good, **bad))
    with pytest.raises(B.AmsError):
        B.ams_assign_pages(**dict(good, table=i32(2, 3), table_out=i32(2, 3)))
