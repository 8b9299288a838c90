"""Caches of 4 bits for the tests: rows, scale bytes and codes written down from their definition in 64 bits, on the host."""
import math

import numpy as np
import torch

from paper_2605_23200_amd import binding as B
from cache_util import BLOCK, DEV, HostCache, blocks

GROUP = 32
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def byte_of(largest: float) -> int:
    if largest == 0:
        return 0
    if not math.isfinite(largest):
        return 255
    e = max(-120, math.frexp(largest)[1] - 5)
    while largest > 7 * 2.0 ** e:
        e += 1
    return e + 127


def power(byte):
    """2^(byte - 127) as float64, NaN for 255."""
    byte = np.asarray(byte).astype(np.float64)
    return np.where(byte == 255, np.nan, 2.0 ** (byte - 127))


def pack_rows(x: np.ndarray):
    """Rows [n, D] float64 -> codes 0 .. 15 [n, D], scale bytes [n, D / 32]."""
    n, D = x.shape
    y = x.reshape(n, D // GROUP, GROUP)
    byte = np.array([[byte_of(float(np.abs(g).max()) if np.isfinite(g).all() else math.inf) for g in row] for row in y], dtype=np.int64)
    byte = byte.reshape(n, D // GROUP)
    usable = (byte > 0) & (byte < 255)
    z = np.where(usable[..., None], y, 0.0) / np.where(usable, power(byte), 1.0)[..., None]
    gap = np.abs(np.abs(z)[..., None] - LEVELS)                              # to every code
    least = gap.min(-1, keepdims=True)
    code = np.where((gap == least) & (np.arange(8) % 2 == 0), 0, np.where(gap == least, 1, 2)).argmin(-1)  # even ones first
    code = code + 8 * (np.signbit(z) & usable[..., None])
    return code.reshape(n, D), byte


def values(codes: np.ndarray, byte: np.ndarray) -> np.ndarray:
    x = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    with np.errstate(invalid="ignore"):
        return x * np.repeat(power(byte), GROUP, -1)


class MicroCache(HostCache):
    """HostCache in 4 bits: t["k"] holds bytes of two codes, t["k_scale"] bytes [..., D / 32, 16]."""

    def __init__(self, shape, capacity, paged=False, seed=0, spare=3):
        super().__init__("int8", shape, capacity, paged, seed, spare)
        self.kind = "e2m1"
        rng = np.random.default_rng(seed + 50)
        for name in ("k", "v"):                          # any byte where no call writes, scales that are no number among them
            self.t[name] = self.t[name][..., :self.D // 2].contiguous().view(torch.uint8)
            lead = tuple(self.t[name + "_scale"].shape)
            self.t[name + "_scale"] = torch.from_numpy(rng.integers(0, 256, lead + (self.D // GROUP, BLOCK), dtype=np.uint8))

    def put(self, name, l, b, h, t, codes, byte):
        rows, at = self.block(name, l, b, h, t // BLOCK)
        rows[t % BLOCK] = torch.from_numpy((codes[0::2] | codes[1::2] << 4).astype(np.uint8))
        self.t[name + "_scale"][at][:, t % BLOCK] = torch.from_numpy(byte.astype(np.uint8))

    def get(self, name, l, b, h, t):
        rows, at = self.block(name, l, b, h, t // BLOCK)
        x = rows[t % BLOCK].numpy().astype(np.int64)
        codes = np.stack([x & 15, x >> 4], -1).reshape(-1)
        return codes, self.t[name + "_scale"][at][:, t % BLOCK].numpy().astype(np.int64)

    def fill(self, name, l, b, h, x):
        codes, byte = pack_rows(x)
        for t in range(len(x)):
            self.put(name, l, b, h, t, codes[t], byte[t])

    def rows(self, name, l, b, h, n):
        out = np.zeros((n, self.D))
        for t in range(n):
            out[t] = values(*self.get(name, l, b, h, t))
        return out

    def copy(self):
        c = MicroCache((self.L, self.B, self.H, self.D), self.capacity, self.paged)
        c.table, c.t = self.table, {k: v.clone() for k, v in self.t.items()}
        return c

    def same_but(self, before, written):
        """Every byte of rows and scales that `written` (a set of (name, l, b, h, t)) does not name is as it was."""
        was = before.copy()
        for name, l, b, h, t in written:
            was.put(name, l, b, h, t, *self.get(name, l, b, h, t))
        for k, v in self.t.items():
            assert torch.equal(v, was.t[k]), k


def filled(shape, capacity, lens, paged=False, seed=0, scale=1.0):
    from cache_util import loud_rows
    c = MicroCache(shape, capacity, paged, seed)
    rng = np.random.default_rng(seed + 100)
    for l in range(c.L):
        for b in range(c.B):
            for h in range(c.H):
                for name in ("k", "v"):
                    c.fill(name, l, b, h, loud_rows(rng, lens[b], c.D) * scale)
    return c
