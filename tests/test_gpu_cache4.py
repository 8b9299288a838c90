"""ams_append, ams_attend, ams_recode and ams_evict over caches of 4 bits against their definitions in 64 bits, and together with
ams_assign_pages as a serving loop calls them.

Tolerances.  Codes, scale bytes, kept positions and copied rows are exact: scales are powers of two and keys that go to 4 bits are
normalised and rotated in 64 bits (1e-15 against half a step of 2^-2: no element here lies that near the middle).  attend: the bounds of
_attend_case, whose steps are the same here: a code times its scale is a bf16 number, so q.k has exact products summed in fp32 and the
second product's operands are exact but for the probabilities' 16 (24) bits."""
import math

import numpy as np
import pytest
import torch

from paper_2605_23200_amd import binding as B
from cache_util import BLOCK, DEV, HostCache, ROWS, as_code_tensor, blocks, lens_dev, loud_rows, pack_block, params, same_bits
from micro_util import GROUP, MicroCache, filled, pack_rows, power, values
from test_gpu_cache import _attend_case, _filled, _kept, _turned

pytestmark = pytest.mark.gpu


def _any(kind, shape, capacity, lens, paged=False, seed=0, scale=1.0):
    return filled(shape, capacity, lens, paged, seed, scale) if kind == "e2m1" else _filled(kind, shape, capacity, lens, paged, seed, scale)


def _clone(c):
    if isinstance(c, MicroCache):
        return c.copy()
    d = HostCache(c.kind, (c.L, c.B, c.H, c.D), c.capacity, c.paged)
    d.table, d.t = c.table, {k: v.clone() for k, v in c.t.items()}
    return d


# ---- ams_recode, ams_evict ----------------------------------------------------------------------------------------

def _check_rows(src, dst, before, pick):
    """dst (downloaded) against the definition; pick(l, b, h) -> source positions (-1: a row of zeros)."""
    written = set()
    for l in range(src.L):
        for b in range(src.B):
            for h in range(src.H):
                idx = pick(l, b, h)
                for name in ("k", "v"):
                    if dst.kind == "e2m1":
                        for j, t in enumerate(idx):
                            if t < 0:
                                want = np.zeros(src.D, np.int64), np.zeros(src.D // GROUP, np.int64)
                            elif src.kind == "e2m1":
                                want = src.get(name, l, b, h, t)     # as they are
                            else:
                                x = src.rows(name, l, b, h, t + 1)[-1:] if src.packed else src.block(name, l, b, h, t // BLOCK)[0][t % BLOCK].double().numpy()[None]
                                want = tuple(y[0] for y in pack_rows(x))
                            got = dst.get(name, l, b, h, j)
                            assert (got[1] == want[1]).all() and (got[0] == want[0]).all(), (name, l, b, h, j, t)
                            written.add((name, l, b, h, j))
                        continue
                    n = max(idx) + 1 if len(idx) and max(idx) >= 0 else 0
                    rows = src.rows(name, l, b, h, n)
                    x = np.stack([rows[t] if t >= 0 else np.zeros(src.D) for t in idx]) if len(idx) else np.zeros((0, src.D))
                    for j in range(blocks(dst.capacity)):
                        got, at = dst.block(name, l, b, h, j)
                        was, _ = before.block(name, l, b, h, j)
                        part = x[j * BLOCK:(j + 1) * BLOCK]
                        if len(part) and dst.packed:
                            codes, scale = pack_block(part, dst.kind)
                            np.testing.assert_equal(float(dst.t[name + "_scale"][at]), scale)
                            same_bits(got[:len(part)], as_code_tensor(codes, dst.kind), "codes")
                        elif len(part):
                            same_bits(got[:len(part)], torch.from_numpy(part).to(torch.float32).to(got.dtype), "rows")
                        same_bits(got[len(part):], was[len(part):], "rows behind the last")
    if dst.kind == "e2m1":
        dst.same_but(before, written)


KINDS = [("bf16", "e2m1"), ("f32", "e2m1"), ("int8", "e2m1"), ("e4m3", "e2m1"), ("e2m1", "bf16"), ("e2m1", "f32"), ("e2m1", "int8"),
         ("e2m1", "e4m3"), ("e2m1", "e2m1")]


def _dtype(*kinds):
    return "f32" if "f32" in kinds else "bf16"


@pytest.mark.parametrize("src_kind,dst_kind", KINDS)
@pytest.mark.parametrize("D,paged_src,paged_dst", [(128, False, True), (64, True, False), (128, True, True)])
def test_recode_whole(src_kind, dst_kind, D, paged_src, paged_dst):
    lens = [0, 1, 16, 37, 70]
    shape = (2, len(lens), 3, D)
    src = _any(src_kind, shape, 70, lens, paged_src, 1)
    dst = _any(dst_kind, shape, 77, [0] * len(lens), paged_dst, 2)
    before = _clone(dst)
    B.ams_recode(params(shape, 70, dtype=_dtype(src_kind, dst_kind)), src.upload(), lens_dev(lens), dst.upload())
    _check_rows(src, dst.download(), before, lambda l, b, h: list(range(lens[b])))


@pytest.mark.parametrize("src_kind,dst_kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_recode_gather(src_kind, dst_kind, D):
    """Rows in any order, twice, outside the cache; counts from none to more than the budget; credit beside them."""
    lens, budget = [200, 131], 83
    shape = (1, 2, 2, D)
    src, dst = _any(src_kind, shape, 200, lens, D == 64, 3), _any(dst_kind, shape, 90, [0, 0], D == 128, 4)
    before = _clone(dst)
    rng = np.random.default_rng(5)
    idx = np.stack([rng.integers(0, lens[u // 2], budget) for u in range(4)]).astype(np.int32)
    idx[0, 7], idx[1, 3], idx[2, 0] = -1, 200, 1 << 30
    n_kept = np.array([budget, 50, 17, 0], np.int32)
    credit = torch.rand((4, 200), device=DEV)
    credit_out = torch.full((4, budget), -3.0, device=DEV)
    B.ams_recode(params(shape, 200, dtype=_dtype(src_kind, dst_kind), budget=budget), src.upload(), None, dst.upload(),
                 torch.from_numpy(idx).to(DEV), torch.from_numpy(n_kept).to(DEV), credit, credit_out)
    inside = lambda t: int(t) if 0 <= t < 200 else -1
    _check_rows(src, dst.download(), before, lambda l, b, h: [inside(t) for t in idx[b * 2 + h, :n_kept[b * 2 + h]]])
    for u in range(4):
        for j in range(budget):
            t = inside(idx[u, j])
            want = credit[u, t] if j < n_kept[u] and t >= 0 else -3.0
            assert float(credit_out[u, j]) == float(want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_recode_values_at_the_edges(dtype):
    """Middles between codes, largest values next to a power's end, subnormals, zeros of both signs, infinities and no number: alone in
    their 32 channels, which they turn; the others keep their values."""
    rng = np.random.default_rng(1)
    x = np.zeros((48, 64))
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0])
    for t in range(48):
        scale = 2.0 ** rng.integers(-40, 40)
        x[t, :32] = np.resize(np.concatenate([mids, -mids]), 32) * scale
        x[t, 32:] = rng.standard_normal(32) * scale
    x[1, :32] *= 1 + 2.0 ** -7                          # 7.05: a power more
    x[2, 5], x[3, 40], x[4, 33] = np.inf, -np.inf, np.nan
    x[5, :32], x[6, 32:] = 0.0, -0.0
    x[7, :32] = 2.0 ** -126 * np.resize([1, 0.5, -0.25, 0], 32)
    x[8, 32:] = 2.0 ** -120 * np.resize([7, 3.5, -0.25, 0.5], 32)
    x[9, :32] = 2.0 ** 126 * np.resize([1.5, -1, 0.25], 32)
    rows = torch.from_numpy(x).to(ROWS[dtype])
    src = HostCache(dtype, (1, 1, 1, 64), 48)
    src.t["k"][0, 0, 0], src.t["v"][0, 0, 0] = rows, rows
    dst, back = MicroCache((1, 1, 1, 64), 48), HostCache(dtype, (1, 1, 1, 64), 48)
    p = params((1, 1, 1, 64), 48, dtype=dtype)
    B.ams_recode(p, src.upload(), lens_dev([48]), dst.upload())
    B.ams_recode(p, B.cache_view(*(dst.dev[n] for n in ("k", "v", "k_scale", "v_scale"))), lens_dev([48]), back.upload())
    dst.download(), back.download()
    codes, byte = pack_rows(rows.double().numpy())
    for t in range(48):
        got = dst.get("k", 0, 0, 0, t)
        assert (got[1] == byte[t]).all() and (got[0] == codes[t]).all(), t
    np.testing.assert_array_equal(back.t["v"][0, 0, 0].double().numpy(), values(codes, byte))
    assert byte[2].tolist()[0] == 255 and byte[3].tolist()[1] == 255 and byte[4].tolist()[1] == 255 and byte[5, 0] == 0


def test_every_code_and_scale_is_read_as_its_value():
    """All 16 codes under every byte, 0 and 255 among them, by ams_recode and, one position a query, by ams_attend."""
    shape, T = (1, 1, 1, 64), 256
    c = MicroCache(shape, T)
    for t in range(T):
        for name in ("k", "v"):
            c.put(name, 0, 0, 0, t, np.tile(np.arange(16), 4), np.array([t, 127]))
    back = HostCache("f32", shape, T)
    B.ams_recode(params(shape, T, dtype="f32"), c.upload(), lens_dev([T]), back.upload())
    back.download()
    want = np.stack([values(*c.get("v", 0, 0, 0, t)) for t in range(T)])
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(back.t["v"][0, 0, 0].numpy(), want.astype(np.float32))
    # sequences of one position each: the output is that position's value
    many = MicroCache((1, T, 1, 64), 1)
    for t in range(T):
        for name in ("k", "v"):
            many.put(name, 0, t, 0, 0, *c.get(name, 0, 0, 0, t))
    p = params((1, T, 1, 64), 1, dtype="f32")
    out, q = torch.zeros((1, T, 1, 1, 64), device=DEV), torch.zeros((1, T, 1, 1, 64), device=DEV)
    ws = torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    B.ams_attend(p, many.upload(), lens_dev([1] * T), q, out, ws)
    got = out.cpu().double().numpy().reshape(T, 64)
    fine = np.arange(T) < 217                           # values below 2^93 (documented for 2^90)
    np.testing.assert_array_equal(got[fine & (np.arange(T) >= 7)], want[fine & (np.arange(T) >= 7)])
    np.testing.assert_allclose(got[:7], want[:7], rtol=0, atol=2.0 ** -124)                      # (bytes that no writer here gives)
    assert np.isnan(got[255]).all()                     # a key that is no number


def test_a_bad_table_entry_is_never_written_through():
    for src_kind, D in (("bf16", 64), ("e2m1", 64), ("e2m1", 128)):
        shape, lens = (1, 2, 2, D), [64, 50]
        src, dst = _any(src_kind, shape, 64, lens, False, 1), filled(shape, 64, [0, 0], True, 2)
        good = dst.table.copy()
        dst.table = good.copy()
        dst.table[0, 1], dst.table[1, 2] = -5, 1 << 20
        before = dst.copy()
        B.ams_recode(params(shape, 64), src.upload(), lens_dev(lens), dst.upload())
        row = torch.ones((1, 2, 1, 2, D), dtype=torch.bfloat16, device=DEV)
        view = B.cache_view(*(dst.dev[n] for n in ("k", "v", "k_scale", "v_scale")), block_table=torch.from_numpy(dst.table).to(DEV))
        B.ams_append(params(shape, 64), None, row, row, None, None, 0.0, None, None, lens_dev([20, 40]), None, view)
        dst.download()
        dst.table = before.table = good
        for b, j in ((0, 1), (1, 2)):
            page = int(good[b, j])
            for name in ("k", "v"):
                assert torch.equal(dst.t[name][:, page * BLOCK:(page + 1) * BLOCK], before.t[name][:, page * BLOCK:(page + 1) * BLOCK])
        spare = sorted(set(range(dst.t["k"].shape[1] // BLOCK)) - set(good.reshape(-1).tolist()))
        for page in spare:
            assert torch.equal(dst.t["k"][:, page * BLOCK:(page + 1) * BLOCK], before.t["k"][:, page * BLOCK:(page + 1) * BLOCK])
            assert torch.equal(dst.t["k_scale"][:, page], before.t["k_scale"][:, page])


@pytest.mark.parametrize("src_kind,dst_kind", [("e2m1", "e2m1"), ("bf16", "e2m1"), ("e2m1", "bf16"), ("int8", "e2m1")])
@pytest.mark.parametrize("D,paged", [(128, True), (64, False)])
def test_evict_types(src_kind, dst_kind, D, paged):
    lens, budget, sink, last = [200, 1, 37, 0, 128], 66, 4, 32
    shape = (2, len(lens), 2, D)
    src, dst = _any(src_kind, shape, 200, lens, paged, 6), _any(dst_kind, shape, 70, [0] * 5, not paged, 7)
    before = _clone(dst)
    units = 2 * 5 * 2
    w = np.random.default_rng(8).random((units, 203)).astype(np.float32)
    w[3, 40:60] = 0.5
    p = params(shape, 200, budget=budget, n_sink=sink, n_last=last, t_stride=203)
    w_out, idx = torch.full((units, 203), -5.0, device=DEV), torch.full((units, budget), -9, dtype=torch.int32, device=DEV)
    n_kept, lens_out = torch.zeros(units, dtype=torch.int32, device=DEV), torch.zeros(5, dtype=torch.int32, device=DEV)
    ws = torch.zeros(B.ams_evict_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    B.ams_evict(p, src.upload(), lens_dev(lens), torch.from_numpy(w).to(DEV), dst.upload(), w_out, idx, n_kept, ws, lens_out)
    want = {u: _kept(w[u], lens[u // 2 % 5], budget, sink, last) for u in range(units)}
    for u in range(units):
        assert idx[u].tolist() == want[u] + [-1] * (budget - len(want[u])) and int(n_kept[u]) == len(want[u])
        assert torch.equal(w_out[u, :len(want[u])].cpu(), torch.from_numpy(w[u, want[u]]))
    assert lens_out.tolist() == [min(n, budget) for n in lens]
    _check_rows(src, dst.download(), before, lambda l, b, h: want[(l * 5 + b) * 2 + h])


# ---- ams_append -----------------------------------------------------------------------------------------------------

def _append_case(dtype, shape, group, lens, n_new, t_max, paged, rope_kw, norm, first, with_q=True, seed=0, loud=1.0):
    L, Bt, H, D = shape
    cache = filled(shape, t_max, lens, paged, seed)
    before = cache.copy()
    rng = np.random.default_rng(seed + 7)
    heads = (group + 2) * H
    qkv = torch.from_numpy(rng.standard_normal((L, Bt, n_new, heads * D + 16)) * loud).to(ROWS[dtype])
    dev = qkv.to(DEV)[..., :heads * D].unflatten(-1, (heads, D))
    q, k, v = dev[..., :group * H, :], dev[..., group * H:(group + 1) * H, :], dev[..., (group + 1) * H:, :]
    host = qkv.double().numpy()[..., :heads * D].reshape(L, Bt, n_new, heads, D)
    w = {n: (torch.from_numpy(1 + 0.3 * rng.standard_normal(D)).to(ROWS[dtype]) if norm else None) for n in "qk"}
    rope = B.make_rope(base=1e4, **rope_kw) if rope_kw else None
    freq = list(rope.freq) if rope else []
    p = params(shape, t_max, group=group, dtype=dtype)
    q_out = torch.full((L, Bt, H * group, n_new, D), -7.0, dtype=ROWS[dtype], device=DEV)
    lens_out = torch.full((Bt,), -9, dtype=torch.int32, device=DEV)
    to_dev = lambda t: t.to(DEV) if t is not None else None
    B.ams_append(p, q if with_q else None, k, v, to_dev(w["q"]), to_dev(w["k"]), 1e-6, rope, lens_dev(first) if first else None, lens_dev(lens),
                 q_out if with_q else None, cache.upload(), lens_out)
    assert lens_out.tolist() == [min(n + n_new, t_max) for n in lens]
    cache.download()
    wd = {n: t.double().numpy() if t is not None else None for n, t in w.items()}
    got_q, gain = q_out.double().cpu().numpy(), abs(rope_kw["gain"]) if rope_kw else 1.0
    written = set()
    for l in range(L):
        for b in range(Bt):
            for t in range(n_new):
                x, pos = host[l, b, t], (first[b] if first else lens[b]) + t
                if with_q:
                    want = _turned(x[:group * H], wd["q"], 1e-6, pos, rope_kw, freq)
                    size = np.abs(want).max(-1, keepdims=True) * 2 + 1e-30       # as in 8 bits: norm, cosine, products in fp32, one rounding
                    bound = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + 16 * 2.0 ** -24 * size * gain
                    assert (np.abs(got_q[l, b, :, t] - want) <= bound).all()
                if lens[b] + t >= t_max:
                    continue
                for name, rows in (("k", _turned(x[group * H:(group + 1) * H], wd["k"], 1e-6, pos, rope_kw, freq)), ("v", x[(group + 1) * H:])):
                    codes, byte = pack_rows(rows)
                    for h in range(H):
                        got = cache.get(name, l, b, h, lens[b] + t)
                        assert (got[1] == byte[h]).all() and (got[0] == codes[h]).all(), (name, l, b, h, t)
                        written.add((name, l, b, h, lens[b] + t))
    cache.same_but(before, written)
    return cache


FULL = dict(rot_dim=128, layout=B.ROPE_HALF, gain=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_new,paged", [(1, False), (1, True), (2, True), (37, False)])
def test_append_types_and_lengths(dtype, n_new, paged):
    """Empty, within a block, at its end; a full sequence takes nothing, one that fills up takes some."""
    _append_case(dtype, (2, 6, 2, 128), 3, [0, 1, 15, 16, 60, 59], n_new, 60, paged, FULL, True, [0, 5, 100000, 1000000, 7, 3])


@pytest.mark.parametrize("layout", [B.ROPE_HALF, B.ROPE_INTERLEAVED])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (128, 40), (128, 2), (128, 6), (128, 90), (64, 64), (64, 24), (64, 10), (64, 0)])
def test_append_layouts(layout, D, rot):
    """Runs of channels that a lane holds fall into the 32 of a scale in every way that the rotations place them."""
    _append_case("bf16", (1, 2, 2, D), 2, [3, 30], 19, 64, False, dict(rot_dim=rot, layout=layout, gain=1.25), True, None)


@pytest.mark.parametrize("norm,with_q,rope,loud", [(False, True, FULL, 1e-30), (True, False, FULL, 1.0), (False, False, None, 1e30)])
def test_append_without_its_parts(norm, with_q, rope, loud):
    _append_case("f32", (1, 2, 3, 128), 2, [14, 33], 5, 64, True, rope, norm, None, with_q, loud=loud)


@pytest.mark.parametrize("heads,group,n_new", [(1, 1, 1), (8, 8, 1), (8, 4, 300)])
def test_append_many_heads_and_tokens(heads, group, n_new):
    _append_case("bf16", (1, 2, heads, 128), group, [5, 77], n_new, 400, True, FULL, True, None, seed=3)


def test_append_token_by_token_is_append_at_once():
    """A row's codes depend on that row alone: whatever the block holds, and in whatever pieces the rows came."""
    shape = (1, 1, 2, 64)
    x = torch.randn((1, 1, 40, 2, 64), device=DEV) * torch.linspace(-8, 8, 40, device=DEV).exp2()[:, None, None]
    x = x.to(torch.bfloat16)
    p = params(shape, 50)
    sides = []
    for pieces in ([40], [1] * 40, [3, 17, 20]):
        c = MicroCache(shape, 50, seed=1)
        view, at = c.upload(), 0
        for n in pieces:
            piece = x[:, :, at:at + n].contiguous()
            B.ams_append(p, None, piece, piece, None, None, 0.0, None, None, lens_dev([at + 5]), None, view)
            at += n
        sides.append(c.download())
    for c in sides[1:]:
        for n in c.t:
            assert torch.equal(c.t[n], sides[0].t[n])


def test_append_no_number_and_infinite():
    """They turn the 32 channels of their row, and no others."""
    shape = (1, 1, 2, 64)
    c = filled(shape, 32, [3])
    before = c.copy()
    k, v = (torch.ones((1, 1, 2, 2, 64), dtype=torch.bfloat16) for _ in range(2))
    k[0, 0, 0, 1, 3], v[0, 0, 1, 0, 63] = math.inf, math.nan
    B.ams_append(params(shape, 32), None, k.to(DEV), v.to(DEV), None, None, 0.0, None, None, lens_dev([3]), None, c.upload())
    c.download()
    one = values(*pack_rows(np.ones((1, 64))))[0]
    for name, h, t, bad in (("k", 1, 3, 0), ("v", 0, 4, 1)):
        codes, byte = c.get(name, 0, 0, h, t)
        assert byte[bad] == 255 and byte[1 - bad] != 255 and not codes[32 * bad:32 * bad + 32].any()
    for name, h, t in (("k", 0, 3), ("k", 1, 4), ("k", 0, 4), ("v", 0, 3), ("v", 1, 3), ("v", 1, 4)):
        np.testing.assert_array_equal(values(*c.get(name, 0, 0, h, t)), one)
    c.same_but(before, {(n, 0, 0, h, t) for n in "kv" for h in (0, 1) for t in (3, 4)})


# ---- ams_attend -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("group,W,causal,paged", [(1, 1, False, False), (4, 1, True, True), (2, 8, True, False), (5, 5, False, True),
                                                 (8, 8, True, False), (7, 11, True, True), (8, 32, True, False), (2, 4, True, True),
                                                 (1, 8, True, False), (7, 1, False, True), (3, 2, True, False)])
def test_attend_shapes(dtype, D, group, W, causal, paged):
    """Every row tile, heads two at a time (up to 8 queries), the two ways to the weights; lengths at the edges of blocks, steps and chunks,
    shorter than the window, empty."""
    lens = [0, 1, 15, 16, 17, 31, 33, 127, 128, 130, 257, 700]
    _attend_case(filled((1, len(lens), 2, D), 701, lens, paged, 5), lens, group, W, dtype, causal, "new", t_stride=705)


@pytest.mark.parametrize("heads", [1, 3, 4])
@pytest.mark.parametrize("group,W", [(4, 1), (2, 4), (3, 5)])
def test_attend_heads_odd_and_even(heads, group, W):
    lens = [300, 77, 0]
    for paged in (False, True):
        _attend_case(filled((2, 3, heads, 128), 305, lens, paged, 15), lens, group, W, causal=True)


@pytest.mark.parametrize("T,heads", [(1, 1), (1, 2), (511, 1), (511, 2), (4100, 1), (4100, 2), (20003, 1), (9001, 2)])
@pytest.mark.parametrize("group,W", [(4, 1), (7, 1), (4, 9)])
def test_attend_lengths_of_one_sequence(T, heads, group, W):
    _attend_case(filled((1, 1, heads, 128), T + 5, [T], False, 6), [T], group, W, causal=True)


@pytest.mark.parametrize("weights,lse", [("new", False), ("same", True), ("zero", True), (None, True), (None, False)])
@pytest.mark.parametrize("W", [1, 7, 20])
def test_attend_outputs_that_are_left_out(weights, lse, W):
    _attend_case(filled((2, 2, 2, 128), 300, [300, 77], False, 7), [300, 77], 2, W, weights=weights, lse=lse)


def test_attend_lengths_outside_the_cache_are_clamped():
    _attend_case(filled((1, 3, 1, 64), 100, [100, 100, 100], False, 8), [5000, -3, 100], 2, 2, causal=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [1, 2])
def test_attend_extreme_scales_and_logits(dtype, heads):
    """Logits of thousands (one position takes all), rows of V 2^60 apart, channels of V 2^50 apart, rows of zeros, an all-zero cache; beside
    an ordinary head."""
    lens = [400] * 4
    cache = filled((1, 4, heads, 128), 400, lens, False, 9)
    rng = np.random.default_rng(2)
    cache.fill("k", 0, 0, 0, loud_rows(rng, 400, 128) * 300)
    v = loud_rows(rng, 400, 128)
    v[100:200] *= 2.0 ** 60
    v[300:] *= 2.0 ** -60
    v[:, 64:] *= 2.0 ** -50
    cache.fill("v", 0, 1, 0, v)
    k, v = loud_rows(rng, 400, 128), loud_rows(rng, 400, 128)
    k[64:128], v[:320] = 0, 0
    cache.fill("k", 0, 2, 0, k)
    cache.fill("v", 0, 2, 0, v)
    cache.fill("k", 0, 3, 0, np.zeros((400, 128)))
    cache.fill("v", 0, 3, 0, np.zeros((400, 128)))
    for W, causal in ((1, False), (2, True), (12, True)):
        _attend_case(cache, lens, 3, W, dtype, causal)


def test_attend_scales_of_another_writer():
    """Codes and scales that the library's writers would not give: any code under any scale, rows far apart, zeros of both signs."""
    shape, lens = (1, 2, 2, 128), [100, 37]
    cache = filled(shape, 160, lens, True, 24)
    rng = np.random.default_rng(9)
    for b in range(2):
        for h in range(2):
            for t in range(lens[b]):
                cache.put("k", 0, b, h, t, rng.integers(0, 16, 128), rng.integers(118, 130, 4))
                cache.put("v", 0, b, h, t, rng.integers(0, 16, 128), rng.integers(60, 190, 4))
    _attend_case(cache, lens, 3, 2, causal=True)
    _attend_case(cache, lens, 3, 9, causal=False)


def test_attend_through_a_bad_table_entry_stays_in_the_pool():
    cache = filled((1, 1, 2, 64), 64, [64], True, 26)
    n_pages = cache.t["k"].shape[1] // BLOCK
    for j in range(n_pages):                            # (spare pages hold any bytes: give every one rows)
        for name in ("k", "v"):
            cache.t[name + "_scale"][:, j] = 127
    p = params((1, 1, 2, 64), 64, group=2)
    q = torch.randn((1, 1, 4, 1, 64), device=DEV).to(torch.bfloat16)
    outs = []
    for entry in (-7, 0, 1 << 30, n_pages - 1):
        cache.table[0, 2] = entry
        out, w = torch.zeros_like(q), torch.zeros((2, 64), device=DEV)
        B.ams_attend(p, cache.upload(), lens_dev([64]), q, out, torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV), None,
                     None, w)
        outs.append((out, w))
    for a, b in ((0, 1), (2, 3)):
        same_bits(outs[a][0], outs[b][0])
        same_bits(outs[a][1], outs[b][1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [3, 4])
@pytest.mark.parametrize("group,W", [(2, 4), (1, 8), (1, 16), (2, 24), (3, 40)])
def test_attend_nan_scales(heads, D, group, W, dtype):
    """32 channels of a key that are no number make the outputs of the queries that see its position NaN; of a value, those 32 outputs of those
    queries; not other queries, heads, channels; not through positions behind the last one, whose bytes may be anything."""
    lens = [160, 147]
    cache = filled((1, 2, heads, D), 200, lens, False, 4)
    bad = {}
    for b, T in enumerate(lens):
        for h, (name, back, part) in enumerate((("k", 3, 0), ("v", 2, D // GROUP - 1), ("v", 7 * 2, 0), ("k", 12, D // GROUP - 1))[:heads]):
            t = T - back
            codes, byte = cache.get(name, 0, b, h, t)
            byte[part] = 255
            codes[part * GROUP:(part + 1) * GROUP] = 0
            cache.put(name, 0, b, h, t, codes, byte)
            bad[b, h] = (name, t, part)
        for h in range(heads):                          # behind the last one: every scale no number
            for t in range(T, blocks(T) * BLOCK):
                for name in ("k", "v"):
                    cache.put(name, 0, b, h, t, np.full(D, 7), np.full(D // GROUP, 255))
    p = params((1, 2, heads, D), 200, group=group, window=W, causal=True, dtype=dtype)
    q = torch.randn((1, 2, heads * group, W, D)).to(ROWS[dtype])
    out = torch.zeros_like(q, device=DEV)
    w = torch.zeros((2 * heads, 200), device=DEV)
    ws = torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    B.ams_attend(p, cache.upload(), lens_dev(lens), q.to(DEV), out, ws, None, None, w)
    nan = torch.isnan(out.float()).cpu()[0]             # [batch, heads * group, W, D]
    for (b, h), (name, t, part) in bad.items():
        sees = torch.arange(W) + lens[b] - W >= t
        channel = torch.ones(D, dtype=torch.bool) if name == "k" else torch.arange(D) // GROUP == part
        want = sees[:, None] & channel[None]
        for g in range(group):
            assert torch.equal(nan[b, h * group + g], want), (b, h, g)
        if name == "v":
            assert not torch.isnan(w[b * heads + h]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("group,W", [(2, 4), (1, 16), (2, 24)])
def test_attend_values_at_the_end_of_the_range(heads, D, group, W, dtype):
    """Scales of 2^126 and 2^127 of V.  Codes under them that are finite count as they are (one step of positions: no probability above 1, no sum
    above the largest value); codes that are not are the business of the queries that see them, not of other queries, channels or heads."""
    lens = [30, 17]
    cache = filled((1, 2, heads, D), 40, lens, heads == 2, 14)
    rng = np.random.default_rng(15)
    for b, t, part, byte in ((0, 28, 0, 254), (0, 27, D // GROUP - 1, 253), (1, 3, 0, 253)):
        codes, scales = cache.get("v", 0, b, heads - 1, t)
        codes[part * GROUP:(part + 1) * GROUP], scales[part] = rng.integers(0, 4, GROUP), byte
        cache.put("v", 0, b, heads - 1, t, codes, scales)
    _attend_case(cache, lens, group, W, dtype, causal=True)

    lens = [160, 147]
    cache = filled((1, 2, heads, D), 200, lens, heads == 2, 16)
    plain, sees = cache.copy(), np.zeros((2, heads, W, D), dtype=bool)
    for b, T in enumerate(lens):
        for h, (back, part, byte) in enumerate(((2, 0, 253), (1, D // GROUP - 1, 254))[:heads]):
            codes, scales = cache.get("v", 0, b, h, T - back)
            codes[part * GROUP:(part + 1) * GROUP], scales[part] = 7, byte
            cache.put("v", 0, b, h, T - back, codes, scales)
            sees[b, h] = (np.arange(W) >= W - back)[:, None]
    p = params((1, 2, heads, D), 200, group=group, window=W, causal=True, dtype=dtype)
    q = torch.randn((1, 2, heads * group, W, D), generator=torch.Generator().manual_seed(3)).to(ROWS[dtype]).to(DEV)
    got = []
    for c in (cache, plain):
        out, w = torch.zeros_like(q), torch.zeros((2 * heads, 200), device=DEV)
        B.ams_attend(p, c.upload(), lens_dev(lens), q, out, torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV), None, None, w)
        got.append((out.cpu().view(2, heads, group, W, D), w))
    # The weights do not know V, but that the sum of a query that sees such a row is (sum - 3/4 y) + y, y = 2^(x + 2), for sum + 2^x: 2^-24 |x + 2|
    # of y from the rounding of x + 2, 2^-22 each of at most 4 sums from the two roundings, where the sum stays.
    logits = max(float(np.abs(q[0, b, h * group:(h + 1) * group].reshape(-1, D).double().cpu().numpy() @ cache.rows("k", 0, b, h, lens[b]).T).max())
                 for b in range(2) for h in range(heads)) / D ** 0.5 * 1.4427
    assert ((got[0][1] - got[1][1]).abs() <= (2.0 ** -24 * (logits + 2) + 2.0 ** -20) * got[1][1]).all()
    for b in range(2):
        for h in range(heads):
            for g in range(group):
                other = torch.from_numpy(~sees[b, h])
                same_bits(got[0][0][b, h, g][other], got[1][0][b, h, g][other])
            # Who sees it: what lies in the other channels is what it was, but for the position's probability (the bits of x + 2, a quarter of the
            # scale: 2^-17 of it in either as two bf16 terms, and less from the exponential) and the rounding of both outputs.
            for g in range(group):
                x, y = got[0][0][b, h, g].double(), got[1][0][b, h, g].double()
                part = slice(GROUP, None) if h == 0 else slice(0, D - GROUP)
                step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -17
                assert ((x - y).abs()[:, part] <= step * y.abs()[:, part] + 2.0 ** -15 * cache_top(plain, b, h, lens[b])).all(), (b, h, g)


def cache_top(cache, b, h, T):
    return float(np.abs(cache.rows("v", 0, b, h, T)).max())


@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("W", [3, 4, 24])
def test_attend_a_query_that_is_no_number(heads, W):
    """The first query of one head's window: its output, its lse and the weights of what it sees; not those of the positions behind it, and
    nothing of the other head."""
    T = 160
    cache = filled((1, 1, heads, 64), 200, [T], False, 4)
    p = params((1, 1, heads, 64), 200, group=2, window=W, causal=True)
    q = torch.randn((1, 1, 2 * heads, W, 64)).to(torch.bfloat16)
    for h in range(heads):
        x = q.clone()
        x[0, 0, 2 * h + 1, 0] = math.nan
        out, lse = torch.zeros_like(q, device=DEV), torch.zeros((1, 1, 2 * heads, W), device=DEV)
        w = torch.zeros((heads, 200), device=DEV)
        ws = torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)
        B.ams_attend(p, cache.upload(), lens_dev([T]), x.to(DEV), out, ws, lse, None, w)
        bad = torch.zeros((2 * heads, W), dtype=torch.bool)
        bad[2 * h + 1, 0] = True
        assert torch.equal(torch.isnan(out.float()).all(-1).cpu()[0, 0], bad) and torch.equal(torch.isnan(out.float()).any(-1).cpu()[0, 0], bad)
        assert torch.equal(torch.isnan(lse).cpu()[0, 0], bad)
        for g in range(heads):
            assert torch.equal(torch.isnan(w[g, :T]).cpu(), torch.arange(T) < (T - W + 1 if g == h else 0))


def test_attend_two_calls_give_the_same_bits():
    cache = filled((2, 2, 4, 128), 1500, [1500, 734], True, 11)
    for W in (1, 20):
        a = _attend_case(cache, [1500, 734], 2, W)
        b = _attend_case(cache, [1500, 734], 2, W)
        for x, y in zip(a, b):
            same_bits(x, y)


def test_pools_beyond_32_bits():
    """Pages whose codes lie past 2^32 bytes of the pool: attended to, appended to, moved."""
    H, D = 8, 128
    n_pages = (1 << 32) // (H * D // 2 * BLOCK) + 300
    shape = (1, 1, H, D)
    small = filled(shape, 100, [100], True, 12)
    far = {}
    shift = n_pages - small.t["k"].shape[1] // BLOCK
    for name in ("k", "v"):
        pool = torch.empty((1, n_pages * BLOCK, H, D // 2), dtype=torch.uint8, device=DEV)
        pool[:, shift * BLOCK:] = small.t[name].to(DEV)
        scale = torch.zeros((1, n_pages, H, D // GROUP, BLOCK), dtype=torch.uint8, device=DEV)
        scale[:, shift:] = small.t[name + "_scale"].to(DEV)
        far[name], far[name + "_scale"] = pool, scale
    table = torch.from_numpy(small.table + shift).to(DEV).to(torch.int32).contiguous()
    view = B.cache_view(far["k"], far["v"], far["k_scale"], far["v_scale"], block_table=table)
    p = params(shape, 100, group=2)
    q = torch.randn((1, 1, 2 * H, 1, D), device=DEV).to(torch.bfloat16)
    row = torch.randn((1, 1, 1, H, D), device=DEV).to(torch.bfloat16)
    outs = []
    for c in (view, small.upload()):
        B.ams_append(p, None, row, row, None, None, 0.0, None, None, lens_dev([99]), None, c)
        out, ws = torch.zeros_like(q), torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)
        w, back = torch.zeros((H, 100), device=DEV), HostCache("bf16", shape, 100)
        B.ams_attend(p, c, lens_dev([100]), q, out, ws, None, None, w)
        B.ams_recode(p, c, lens_dev([100]), back.upload())
        outs.append((out, w, back.dev["k"], back.dev["v"]))
    for x, y in zip(*outs):
        same_bits(x, y)


def test_slabs_of_very_many_rows():
    """Slabs so long that the way from one head to the next is almost 2^30 bytes (heads two at a time), and that long (one at a time)."""
    H, D, T = 2, 128, 300
    small = filled((1, 1, H, D), 304, [T], False, 30)
    q = torch.randn((1, 1, 3 * H, 1, D), device=DEV).to(torch.bfloat16)
    row = torch.randn((1, 1, 1, H, D), device=DEV).to(torch.bfloat16)
    p = params((1, 1, H, D), 304, group=3)
    outs = []
    for rows in (304, (1 << 24) - 16, 1 << 24):
        t = {}
        for name in ("k", "v"):
            t[name] = torch.empty((1, 1, H, rows, D // 2), dtype=torch.uint8, device=DEV)
            t[name][:, :, :, :304] = small.t[name].to(DEV)
            t[name + "_scale"] = torch.empty((1, 1, H, rows // BLOCK, D // GROUP, BLOCK), dtype=torch.uint8, device=DEV)
            t[name + "_scale"][:, :, :, :19] = small.t[name + "_scale"].to(DEV)
        view = B.cache_view(t["k"], t["v"], t["k_scale"], t["v_scale"])
        B.ams_append(p, None, row, row, None, None, 0.0, None, None, lens_dev([T]), None, view)
        out, w = torch.zeros_like(q), torch.zeros((H, 304), device=DEV)
        B.ams_attend(p, view, lens_dev([T + 1]), q, out, torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV), None, None, w)
        outs.append((out.float(), w))
        del t, view
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    # the other kernel sums in another order: two roundings to bf16 of the same value may differ by one step, weights by the bound of a probability
    assert (outs[0][0] - outs[2][0]).abs().max() <= 2.0 ** -7 * outs[0][0].abs().max()
    assert ((outs[0][1] - outs[2][1]).abs() <= 2.0 ** -14 * outs[0][1] + 1e-30).all()


# ---- together ---------------------------------------------------------------------------------------------------------

class _Loop:
    """A serving loop over a pool of 4 bits: pages follow the lengths, tokens go in, are attended to, caches go back to their budget; all on
    the device.  `pool`: block tables by ams_assign_pages; else slabs of the same capacity."""
    L, H, G, D, CAP, BUDGET = 2, 2, 3, 64, 96, 48

    def __init__(self, batch, pool, seed=0):
        self.B, self.pool = batch, pool
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.r = lambda *s: torch.randn(s, generator=gen, device=DEV).to(torch.bfloat16)
        self.i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        shape = (self.L, batch, self.H, self.D)
        self.p = params(shape, self.CAP, group=self.G, budget=self.BUDGET, n_sink=2, n_last=8)
        self.rope = B.make_rope(self.D)
        self.width = blocks(self.CAP)
        self.n_pages = batch * self.width * 2
        u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV)
        self.tables = [torch.full((batch, self.width), -1, dtype=torch.int32, device=DEV) for _ in range(2)]
        if pool:
            lead, scales = (self.L, self.n_pages * BLOCK, self.H), (self.L, self.n_pages, self.H, self.D // GROUP, BLOCK)
            t = [u8(*lead, self.D // 2), u8(*lead, self.D // 2), u8(*scales), u8(*scales)]
            self.views = [B.cache_view(*t, block_table=table) for table in self.tables]
        else:
            lead = (self.L, batch, self.H, self.CAP)
            scales = lead[:3] + (self.width, self.D // GROUP, BLOCK)
            self.views = [B.cache_view(u8(*lead, self.D // 2), u8(*lead, self.D // 2), u8(*scales), u8(*scales)) for _ in range(2)]
        self.ring = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV)
        self.state = [torch.tensor([0, self.n_pages], dtype=torch.int32, device=DEV), self.i32(2)]
        units = self.L * batch * self.H
        self.weights = [torch.zeros((units, self.CAP), device=DEV) for _ in range(2)]
        self.lens, self.none = self.i32(batch), self.i32(batch)
        self.idx, self.n_kept = self.i32(units, self.BUDGET), self.i32(units)
        self.ws = torch.empty(B.ams_attend_workspace_bytes(self.p), dtype=torch.uint8, device=DEV)
        self.ws_evict = torch.empty(B.ams_evict_workspace_bytes(self.p), dtype=torch.uint8, device=DEV)

    def assign(self, table, to, slots=None):
        if self.pool:
            lens_out = torch.empty_like(self.lens)
            B.ams_assign_pages(self.p, self.lens if table is self.tables[0] or slots is not None else self.none, to, table, table, self.ring,
                               self.state[0], self.state[1], None, slots, lens_out)
            self.state.reverse()
            return lens_out
        return to.clone()

    def step(self, x):
        """x [L, B, new, heads, D] a projection's output; returns the attention of the new tokens."""
        new, HQ = x.shape[2], self.H * self.G
        slots = torch.zeros(self.B * new + 3, dtype=torch.int64, device=DEV)
        to = self.assign(self.tables[0], self.lens + new, slots)
        q = torch.empty((self.L, self.B, HQ, new, self.D), dtype=torch.bfloat16, device=DEV)
        after = torch.empty_like(self.lens)
        B.ams_append(self.p, x[..., :HQ, :], x[..., HQ:HQ + self.H, :], x[..., HQ + self.H:, :], None, None, 0.0, self.rope, self.lens, self.lens, q,
                     self.views[0], after)
        self.lens = after
        p = params((self.L, self.B, self.H, self.D), self.CAP, group=self.G, window=new, causal=True)
        ws = torch.empty(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)
        out = torch.empty_like(q)
        B.ams_attend(p, self.views[0], self.lens, q, out, ws, None, self.weights[0], self.weights[0])
        return out, to, slots

    def bound(self):
        """Back to the budget: pages for what stays, the move, the old pages back."""
        keep = self.lens.clamp(max=self.BUDGET)
        self.assign(self.tables[1], keep)
        after = torch.empty_like(self.lens)
        B.ams_evict(self.p, self.views[0], self.lens, self.weights[0], self.views[1], self.weights[1], self.idx, self.n_kept, self.ws_evict, after)
        self.assign(self.tables[0], self.none)
        for pair in (self.tables, self.views, self.weights):
            pair.reverse()
        self.lens = after

    def end(self, which):
        """Requests that are done give their pages back; their lengths and weights become 0."""
        to = torch.where(which, 0, self.lens)
        self.assign(self.tables[0], to)
        self.lens = to
        self.weights[0][which.repeat_interleave(self.H).repeat(self.L)] = 0


def _script(loop):
    outs = [loop.step(loop.r(loop.L, loop.B, 30, (loop.G + 2) * loop.H, loop.D))]
    for t in range(64):
        outs.append(loop.step(loop.r(loop.L, loop.B, 1, (loop.G + 2) * loop.H, loop.D)))
        if t in (20, 45):
            loop.bound()
        if t == 33:
            loop.end(torch.arange(loop.B, device=DEV) % 2 == 0)
    return outs


def test_a_serving_loop_over_pages_is_one_over_slabs():
    """The same bits, and at every point no page with two sequences or with one and in the ring."""
    paged, dense = _Loop(5, True), _Loop(5, False)
    a, b = _script(paged), _script(dense)
    for (x, to, slots), (y, want, _) in zip(a, b):
        same_bits(x, y)
        assert torch.equal(to, want)
    same_bits(paged.weights[0], dense.weights[0])
    head, count = paged.state[0].tolist()
    free = [int(paged.ring[(head + i) % paged.n_pages]) for i in range(count)]
    used = [int(v) for b, n in enumerate(paged.lens.tolist()) for v in paged.tables[0][b, :blocks(n)]]
    assert sorted(free + used) == list(range(paged.n_pages))
    assert (paged.tables[1] == -1).all()
    slots = a[-1][2].tolist()                           # of the last step: every sequence's newest position
    last = [int(paged.tables[0][b, (n - 1) // BLOCK]) * BLOCK + (n - 1) % BLOCK for b, n in enumerate(paged.lens.tolist())]
    assert slots == last + [-1] * 3


def test_a_captured_step_replays():
    """A step of the loop in a graph, its lengths and ring carried on in place: the same bits as eager, replay by replay."""
    eager, loop = _Loop(4, True, 3), _Loop(4, True, 3)
    first = eager.r(2, 4, 30, 10, 64)
    loop.step(first), eager.step(first)
    tokens = [eager.r(2, 4, 1, 10, 64) for _ in range(12)]
    x = tokens[0].clone()
    lens, state = loop.lens, loop.state[0]
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    keep = {k: v.clone() for k, v in dict(lens=lens, state=state, ring=loop.ring, table=loop.tables[0], w=loop.weights[0]).items()}
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        out, to, slots = loop.step(x)
        lens.copy_(loop.lens)
        state.copy_(loop.state[0])
    for name, t in (("lens", lens), ("state", state), ("ring", loop.ring), ("table", loop.tables[0]), ("w", loop.weights[0])):
        assert torch.equal(t, keep[name])               # nothing ran yet
    for i, token in enumerate(tokens):
        want, want_to, want_slots = eager.step(token)
        x.copy_(token)
        graph.replay()
        torch.cuda.synchronize()
        same_bits(out, want)
        assert torch.equal(to, want_to) and torch.equal(slots, want_slots), i
        assert torch.equal(loop.tables[0], eager.tables[0]) and torch.equal(state, eager.state[0]) and torch.equal(lens, eager.lens)
        same_bits(loop.weights[0], eager.weights[0])


def test_two_streams_at_once():
    cache = filled((1, 2, 4, 128), 1000, [1000] * 2, False, 21)
    view, lens = cache.upload(), lens_dev([1000] * 2)
    p = params((1, 2, 4, 128), 1000, group=4)
    jobs = []
    for i in range(2):
        q = torch.randn((1, 2, 16, 1, 128), device=DEV).to(torch.bfloat16)
        jobs.append(dict(q=q, out=torch.zeros_like(q), w=torch.zeros((8, 1000), device=DEV), stream=torch.cuda.Stream(),
                         ws=torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)))
    alone = []
    for j in jobs:
        B.ams_attend(p, view, lens, j["q"], j["out"], j["ws"], None, None, j["w"])
        alone.append((j["out"].clone(), j["w"].clone()))
    torch.cuda.synchronize()
    for _ in range(5):
        for j in jobs:
            with torch.cuda.stream(j["stream"]):
                B.ams_attend(p, view, lens, j["q"], j["out"], j["ws"], None, None, j["w"])
    torch.cuda.synchronize()
    for j, (out, w) in zip(jobs, alone):
        same_bits(j["out"], out)
        same_bits(j["w"], w)


def test_binding_types():
    """The tensors that a cache of 4 bits is made of, and those that it is not."""
    c = filled((1, 1, 2, 64), 40, [40], False, 22)
    view = c.upload()
    t = c.dev
    other = B.cache_view(*(t[n].view(torch.float4_e2m1fn_x2) for n in ("k", "v")), *(t[n].view(torch.float8_e8m0fnu) for n in ("k_scale", "v_scale")))
    p = params((1, 1, 2, 64), 40, group=2)
    q = torch.randn((1, 1, 4, 1, 64), device=DEV).to(torch.bfloat16)
    outs = []
    for v in (view, other):
        out, ws = torch.zeros_like(q), torch.zeros(B.ams_attend_workspace_bytes(p), dtype=torch.uint8, device=DEV)
        B.ams_attend(p, v, lens_dev([40]), q, out, ws)
        outs.append(out)
    same_bits(*outs)
    scale = t["k_scale"]
    for args in ((t["k"], t["v"]), (t["k"], t["v"], scale, scale[:, :, :, :2].contiguous()), (t["k"], t["v"], scale.float(), scale.float()),
                 (t["k"], t["v"], scale.transpose(-1, -2).contiguous(), scale), (t["k"], t["v"].view(torch.int8), scale, scale),
                 (t["k"], t["v"], scale.cpu(), scale)):
        with pytest.raises(ValueError):
            B.cache_view(*args)
    with pytest.raises(ValueError):                     # 128 channels asked of rows of 32 bytes
        B.ams_attend(params((1, 1, 2, 128), 40, group=2), view, lens_dev([40]), q, torch.zeros_like(q), ws)
