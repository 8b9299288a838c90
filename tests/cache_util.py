"""Caches of 8 bits for the tests: blocks, scales and codes written down from their definition in 64 bits, on the host."""
import math

import numpy as np
import torch

from paper_2605_23200_amd import binding as B

DEV = "cuda:0"
BLOCK = 16
MOST = {"int8": 127.0, "e4m3": 448.0}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
ROWS = {"bf16": torch.bfloat16, "f32": torch.float32}
KV = {"bf16": B.BF16, "f32": B.F32}


def blocks(n):
    return -(-n // BLOCK)


def scale_of(largest: float, kind: str) -> float:
    if largest == 0:
        return 0.0
    if not math.isfinite(largest):
        return math.nan
    e = -120
    while largest > MOST[kind] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def round_codes(y: np.ndarray, kind: str) -> np.ndarray:
    """float64 values / scale -> values of the nearest codes, ties to even."""
    if kind == "int8":
        return np.rint(y)
    a = np.abs(y)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.rint(y / step) * step


def pack_block(x: np.ndarray, kind: str, had: float = 0.0):
    """Rows [n, D] of one block -> (values of their codes, scale); had: the scale of rows that are there already."""
    need = scale_of(float(np.abs(x).max()) if np.isfinite(x).all() else math.inf, kind)
    scale = math.nan if math.isnan(need) or math.isnan(had) else max(need, had)
    if not scale > 0:
        return np.zeros_like(x), scale
    return round_codes(x / scale, kind), scale


def as_code_tensor(values: np.ndarray, kind: str) -> torch.Tensor:
    return torch.from_numpy(values.astype(np.float32)).to(CODE[kind])


class HostCache:
    """Rows [L, Bt, H, T, D] in float64 or codes and scales, dense or paged; on the GPU through `upload`."""

    def __init__(self, kind, shape, capacity, paged=False, seed=0, spare=3):
        self.kind, self.paged = kind, paged
        self.L, self.B, self.H, self.D = shape
        self.capacity = capacity
        self.packed = kind in CODE
        rng = np.random.default_rng(seed)
        dtype = CODE[kind] if self.packed else ROWS[kind]
        if paged:
            nb = blocks(capacity)
            n_pages = self.B * nb + spare
            self.table = rng.permutation(n_pages)[:self.B * nb].reshape(self.B, nb).astype(np.int32)
            lead = (self.L, n_pages * BLOCK, self.H)
            scales = (self.L, n_pages, self.H)
        else:
            self.table = None
            lead = (self.L, self.B, self.H, capacity)
            scales = (self.L, self.B, self.H, blocks(capacity))
        self.t = {}
        for name in ("k", "v"):
            if self.packed:
                # what no call may take for data: any byte, codes that are no number among them
                raw = torch.from_numpy(rng.integers(0, 256, lead + (self.D,), dtype=np.uint8)).view(dtype)
                self.t[name + "_scale"] = torch.full(scales, 7.0)
            else:
                raw = torch.full(lead + (self.D,), math.nan, dtype=dtype)
            self.t[name] = raw

    def block(self, name, l, b, h, j):
        """(view of the codes' rows [16 or fewer, D], index of the scale)"""
        if self.paged:
            page = int(self.table[b, j])
            return self.t[name][l, page * BLOCK:(page + 1) * BLOCK, h], (l, page, h)
        return self.t[name][l, b, h, j * BLOCK:(j + 1) * BLOCK], (l, b, h, j)

    def fill(self, name, l, b, h, x: np.ndarray):
        """Rows 0 .. n of one unit from float64."""
        for j in range(blocks(len(x))):
            part = x[j * BLOCK:(j + 1) * BLOCK]
            rows, at = self.block(name, l, b, h, j)
            if self.packed:
                codes, scale = pack_block(part, self.kind)
                rows.view(torch.uint8)[:len(part)] = as_code_tensor(codes, self.kind).view(torch.uint8)
                self.t[name + "_scale"][at] = scale
            else:
                rows[:len(part)] = torch.from_numpy(part).to(rows.dtype)

    def rows(self, name, l, b, h, n) -> np.ndarray:
        """Rows 0 .. n as float64."""
        out = np.zeros((n, self.D))
        for j in range(blocks(n)):
            rows, at = self.block(name, l, b, h, j)
            m = min(BLOCK, n - j * BLOCK)
            x = rows[:m].to(torch.float32).double().numpy()
            if self.packed:
                with np.errstate(invalid="ignore"):
                    x = x * float(self.t[name + "_scale"][at])
            out[j * BLOCK:j * BLOCK + m] = x
        return out

    def upload(self):
        d = {k: v.to(DEV) for k, v in self.t.items()}
        self.dev = d
        table = torch.from_numpy(self.table).to(DEV) if self.paged else None
        return B.cache_view(d["k"], d["v"], d.get("k_scale"), d.get("v_scale"), block_table=table)

    def download(self):
        for k, v in self.dev.items():
            self.t[k] = v.cpu()
        return self


def bits(t: torch.Tensor) -> np.ndarray:
    return t.cpu().contiguous().view(torch.uint8).numpy()


def same_bits(a: torch.Tensor, b: torch.Tensor, what=""):
    x, y = bits(a), bits(b)
    assert x.shape == y.shape and (x == y).all(), f"{what}: {(x != y).sum()} of {x.size} bytes differ"


def params(cache_or_shape, t_max, *, group=1, window=1, dtype="bf16", **kw):
    L, Bt, H, D = cache_or_shape
    return B.make_params(n_layers=L, batch=Bt, n_kv_heads=H, group=group, window=window, head_dim=D, kv_dtype=KV[dtype], t_max=t_max,
                         budget=kw.pop("budget", t_max), n_segments=1, **kw)


def lens_dev(lens):
    return torch.tensor(lens, dtype=torch.int32, device=DEV)


def loud_rows(rng, n, d):
    """Rows of different loudness with a loud channel; what a bf16 cache can hold."""
    x = rng.standard_normal((n, d)) * np.exp(0.5 * rng.standard_normal((n, 1)))
    x[:, d // 3] *= 4
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()
