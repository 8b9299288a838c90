"""Thin Python face of the C-ABI library (include/ams.h): argument marshalling only.

Every function has the name and the argument order of its C entry point, takes torch tensors that
live on the GPU (PyTorch is used for device memory and streams, nothing else), passes their raw
pointers through ctypes and raises on a non-zero status.  There is no CPU fallback: if the built
library is missing, importing the entry points fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libams.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_HIP = 0, 1, 2, 3, 4
F32, BF16 = 0, 1
INT8, E4M3, E2M1 = 2, 3, 4            # element types of a cache only (cache_view)
SCORER_LAST_QUERY, SCORER_MEAN_WINDOW, SCORER_KEYDIFF, SCORER_EXPECTED, SCORER_EXTERNAL = 0, 1, 2, 3, 4
SCORER_EXPECTED_VNORM = 5
SCORER_REDUNDANCY = 6
LAYOUT_DENSE, LAYOUT_PAGED = 0, 1
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = 0, 1, 2, 3
SCORE_PATH_AUTO, SCORE_PATH_TWO_SWEEPS, SCORE_PATH_ONE_READ, SCORE_PATH_ONE_LAUNCH = 0, 1, 2, 3

EXPORTS = ("ams_status_string", "ams_workspace_bytes", "ams_workspace_layout", "ams_profile_begin",
           "ams_profile_end", "ams_debug_set_wait_limit", "ams_score",
           "ams_ema_update", "ams_mass_segment", "ams_mass_segment_static", "ams_select", "ams_compact",
           "ams_compress_step", "ams_rope_init", "ams_append", "ams_attend_workspace_bytes", "ams_attend", "ams_recode",
           "ams_evict_workspace_bytes", "ams_evict", "ams_assign_pages")


class AmsError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


class Params(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("batch", C.c_int32), ("n_kv_heads", C.c_int32),
                ("group", C.c_int32), ("head_dim", C.c_int32), ("window", C.c_int32),
                ("kv_dtype", C.c_int32), ("t_max", C.c_int32), ("t_stride", C.c_int64),
                ("budget", C.c_int32), ("n_segments", C.c_int32), ("q_min", C.c_int32),
                ("ema_lambda", C.c_float), ("ema_beta", C.c_float), ("mass_eps", C.c_float),
                ("scorer", C.c_int32), ("n_sink", C.c_int32), ("n_last", C.c_int32), ("causal", C.c_int32),
                ("seg_delta", C.c_float), ("l_min", C.c_int32), ("l_max", C.c_int32), ("pool_kernel", C.c_int32),
                ("vnorm_eps", C.c_float), ("score_path", C.c_int32),
                ("mix_lambda", C.c_float), ("score_kernel", C.c_int32)]

    @property
    def units(self) -> int:
        return self.n_layers * self.batch * self.n_kv_heads


class KvView(C.Structure):
    _fields_ = [("layout", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("t_capacity", C.c_int64),
                ("block_table", C.c_void_p), ("max_blocks_per_seq", C.c_int32), ("block_size", C.c_int32),
                ("n_slots", C.c_int64)]


class WorkspaceView(C.Structure):
    _fields_ = [("u", C.c_size_t), ("g", C.c_size_t), ("m_used", C.c_size_t), ("bounds", C.c_size_t),
                ("seg_mass", C.c_size_t), ("quota", C.c_size_t)]


class Cache(C.Structure):
    """A cache of any element type (cache_view).  Keeps its tensors alive; `index` is their GPU."""
    _fields_ = [("kv", KvView), ("dtype", C.c_int32), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class Rope(C.Structure):
    _fields_ = [("layout", C.c_int32), ("rot_dim", C.c_int32), ("gain", C.c_float), ("freq", C.c_double * 64)]


class NewTokens(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("norm_eps", C.c_float),
                ("positions", C.c_void_p), ("n_new", C.c_int32)]


class Pages(C.Structure):
    _fields_ = [("table", C.c_void_p), ("table_out", C.c_void_p), ("max_blocks_per_seq", C.c_int32), ("n_pages", C.c_int32),
                ("ring", C.c_void_p), ("state", C.c_void_p), ("state_out", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """Loads the built library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2605_23200_amd.build` "
                              "(or __graft_entry__.build()) first")
        l = C.CDLL(LIB_PATH)
        l.ams_status_string.restype = C.c_char_p
        l.ams_status_string.argtypes = [C.c_int]
        l.ams_workspace_bytes.restype = C.c_size_t
        l.ams_workspace_bytes.argtypes = [C.POINTER(Params)]
        l.ams_workspace_layout.argtypes = [C.POINTER(Params), C.POINTER(WorkspaceView)]
        P, V, p = C.POINTER(Params), C.POINTER(KvView), C.c_void_p
        l.ams_score.argtypes = [P, V, p, p, p, p, p, C.c_size_t, p]
        l.ams_ema_update.argtypes = [P, p, p, p, p, p, C.c_size_t, p]
        l.ams_mass_segment.argtypes = [P, p, p, p, p, p, C.c_size_t, p]
        l.ams_mass_segment_static.argtypes = [P, p, p, p, p, p]
        l.ams_select.argtypes = [P, p, p, p, p, p, p, p, p, C.c_size_t, p]
        l.ams_compact.argtypes = [P, V, p, p, V, p, p, p]
        l.ams_compress_step.argtypes = [P, V, p, p, p, V, p, p, p, p, C.c_size_t, p]
        l.ams_profile_end.argtypes = [p, C.c_int, C.POINTER(C.c_char_p), C.POINTER(C.c_float)]
        K, d = C.POINTER(Cache), C.c_double
        l.ams_rope_init.argtypes = [C.POINTER(Rope), C.c_int32, C.c_int32, d, C.c_int32, d, C.c_int32, d, d, C.c_float]
        l.ams_append.argtypes = [P, C.POINTER(NewTokens), C.POINTER(Rope), p, p, K, p, p]
        l.ams_attend.argtypes = [P, K, p, p, p, p, p, p, p, C.c_size_t, p]
        l.ams_recode.argtypes = [P, K, p, p, p, K, p, p, p]
        l.ams_evict.argtypes = [P, K, p, p, K, p, p, p, p, p, C.c_size_t, p]
        l.ams_assign_pages.argtypes = [P, C.POINTER(Pages), p, p, p, p, p, C.c_int64, p]
        for name in EXPORTS[2:]:
            getattr(l, name).restype = C.c_int
        for name in ("ams_attend_workspace_bytes", "ams_evict_workspace_bytes"):
            getattr(l, name).restype = C.c_size_t
            getattr(l, name).argtypes = [P]
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().ams_status_string(int(status)).decode()


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return C.c_void_p(t.data_ptr())


def _stream(stream) -> C.c_void_p:
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _check(rc: int, what: str):
    if rc != OK:
        raise AmsError(rc, what)


def make_params(*, n_layers, batch, n_kv_heads, group, window, head_dim=128, kv_dtype=BF16, t_max,
                t_stride=None, budget, n_segments, q_min=1, ema_lambda=0.9, ema_beta=0.9, mass_eps=1e-6,
                scorer=SCORER_MEAN_WINDOW, n_sink=0, n_last=0, causal=False, seg_delta=0.0, l_min=0, l_max=0,
                pool_kernel=0, vnorm_eps=1e-2, score_path=SCORE_PATH_AUTO,
                mix_lambda=0.07, score_kernel=7) -> Params:
    return Params(n_layers, batch, n_kv_heads, group, head_dim, window, kv_dtype, t_max,
                  t_stride if t_stride is not None else t_max, budget, n_segments, q_min,
                  ema_lambda, ema_beta, mass_eps, scorer, int(n_sink), int(n_last), int(bool(causal)),
                  float(seg_delta), int(l_min), int(l_max), int(pool_kernel), float(vnorm_eps), int(score_path),
                  float(mix_lambda), int(score_kernel))


def dense_view(k: torch.Tensor, v: Optional[torch.Tensor]) -> KvView:
    """k, v: [L, B, H, t_capacity, D] device tensors (any 2- or 4-byte element type)."""
    assert k.dim() == 5
    return KvView(LAYOUT_DENSE, k.data_ptr(), v.data_ptr() if v is not None else None, k.shape[3],
                  None, 0, 0, 0)


def paged_view(k_pool: torch.Tensor, v_pool: Optional[torch.Tensor], block_table: torch.Tensor,
               block_size: int = 16) -> KvView:
    """k_pool, v_pool: [L, n_slots, H, D]; block_table: int32 [B, max_blocks]."""
    assert k_pool.dim() == 4 and block_table.dtype == torch.int32 and block_table.is_contiguous()
    return KvView(LAYOUT_PAGED, k_pool.data_ptr(), v_pool.data_ptr() if v_pool is not None else None, 0,
                  block_table.data_ptr(), block_table.shape[1], block_size, k_pool.shape[1])


def ams_workspace_bytes(p: Params) -> int:
    return int(lib().ams_workspace_bytes(C.byref(p)))


def ams_workspace_layout(p: Params) -> WorkspaceView:
    out = WorkspaceView()
    _check(lib().ams_workspace_layout(C.byref(p), C.byref(out)), "ams_workspace_layout")
    return out


def ams_profile_begin():
    _check(lib().ams_profile_begin(), "ams_profile_begin")


def ams_debug_set_wait_limit(polls: int):
    _check(lib().ams_debug_set_wait_limit(int(polls)), "ams_debug_set_wait_limit")


def ams_profile_end(stream=None, max_entries: int = 4096):
    """Returns [(kernel label, milliseconds), ...] in launch order; waits for the stream."""
    labels = (C.c_char_p * max_entries)()
    ms = (C.c_float * max_entries)()
    n = lib().ams_profile_end(_stream(stream), max_entries, labels, ms)
    if n < 0:
        raise AmsError(-n, "ams_profile_end")
    return [(labels[i].decode(), float(ms[i])) for i in range(n)]


def ams_score(p, src, seq_lens, q, u, g, ws, stream=None):
    _check(lib().ams_score(C.byref(p), C.byref(src), _ptr(seq_lens), _ptr(q), _ptr(u), _ptr(g), _ptr(ws),
                           ws.numel() * ws.element_size(), _stream(stream)), "ams_score")


def ams_ema_update(p, seq_lens, u, credit, m_used, ws=None, stream=None):
    _check(lib().ams_ema_update(C.byref(p), _ptr(seq_lens), _ptr(u), _ptr(credit), _ptr(m_used), _ptr(ws),
                                ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)),
           "ams_ema_update")


def ams_mass_segment(p, seq_lens, m_used, bounds, seg_mass, ws=None, stream=None):
    _check(lib().ams_mass_segment(C.byref(p), _ptr(seq_lens), _ptr(m_used), _ptr(bounds), _ptr(seg_mass),
                                  _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0,
                                  _stream(stream)), "ams_mass_segment")


def ams_mass_segment_static(p, seq_lens, m_used, bounds, seg_mass, stream=None):
    _check(lib().ams_mass_segment_static(C.byref(p), _ptr(seq_lens), _ptr(m_used), _ptr(bounds), _ptr(seg_mass),
                                         _stream(stream)), "ams_mass_segment_static")


def ams_select(p, seq_lens, g, bounds, seg_mass, quota, idx, n_kept, ws=None, stream=None):
    _check(lib().ams_select(C.byref(p), _ptr(seq_lens), _ptr(g), _ptr(bounds), _ptr(seg_mass), _ptr(quota),
                            _ptr(idx), _ptr(n_kept), _ptr(ws),
                            ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)),
           "ams_select")


def ams_compact(p, src, idx, n_kept, dst, credit_src=None, credit_dst=None, stream=None):
    _check(lib().ams_compact(C.byref(p), C.byref(src), _ptr(idx), _ptr(n_kept), C.byref(dst),
                             _ptr(credit_src), _ptr(credit_dst), _stream(stream)), "ams_compact")


def ams_compress_step(p, src, seq_lens, q, credit, dst, credit_dst, idx, n_kept, ws, stream=None):
    _check(lib().ams_compress_step(C.byref(p), C.byref(src), _ptr(seq_lens), _ptr(q), _ptr(credit),
                                   C.byref(dst), _ptr(credit_dst), _ptr(idx), _ptr(n_kept), _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream(stream)), "ams_compress_step")


# ---- between two events: new rows, attention, eviction, caches in 8 and 4 bits, pages ----

def _types(*names):
    """Those of torch's types that this torch has (those of 4 bits and of their scales came late; uint8 stands for either)."""
    return tuple(getattr(torch, n) for n in names if hasattr(torch, n))


_CACHE_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.int8: INT8, torch.float8_e4m3fn: E4M3,
                 **dict.fromkeys(_types("uint8", "float4_e2m1fn_x2"), E2M1)}
_SCALE_DTYPES = {INT8: (torch.float32,), E4M3: (torch.float32,), E2M1: _types("uint8", "float8_e8m0fnu")}
BLOCK = 16                             # positions that share a scale (in 4 bits: whose scales lie together); a page
MICRO = 32                             # channels of a row that share a scale in 4 bits


def scale_shape(k: torch.Tensor):
    """Shape of k_scale and v_scale of a cache whose keys have the shape of `k` (dense or paged; in 4 bits two channels an element)."""
    lead = tuple(k.shape[:3]) + (-(-k.shape[3] // BLOCK),) if k.dim() == 5 else (k.shape[0], k.shape[1] // BLOCK, k.shape[2])
    return lead + (2 * k.shape[-1] // MICRO, BLOCK) if _CACHE_DTYPES.get(k.dtype) == E2M1 else lead


def cache_view(k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
               v_scale: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None) -> Cache:
    """A cache of rows (bf16, fp32) or of codes (int8, float8_e4m3fn; two a byte in uint8 or float4_e2m1fn_x2) with their scales: k, v
    [L, B, H, t_capacity, D], or, with a block table (int32 [B, max_blocks]), pools [L, n_slots, H, D]; D / 2 bytes a row in 4 bits."""
    tensors = [t for t in (k, v, k_scale, v_scale, block_table) if t is not None]
    if any(not t.is_cuda or t.device != k.device for t in tensors):
        raise ValueError("a cache's tensors lie on one GPU")
    if any(not t.is_contiguous() for t in tensors):
        raise ValueError("contiguous tensor expected")
    if k.dtype not in _CACHE_DTYPES or k.dtype != v.dtype or k.shape != v.shape or k.dim() != (5 if block_table is None else 4):
        raise ValueError("k and v: one shape, one element type of bf16, fp32, int8, float8_e4m3fn, uint8, float4_e2m1fn_x2; "
                         "five dimensions, paged four")
    dtype = _CACHE_DTYPES[k.dtype]
    if dtype in _SCALE_DTYPES:
        kinds = _SCALE_DTYPES[dtype]
        for t in (k_scale, v_scale):
            if t is None or t.dtype not in kinds or tuple(t.shape) != scale_shape(k):
                raise ValueError(f"{' or '.join(str(t) for t in kinds)} scales of shape {scale_shape(k)} expected")
    elif k_scale is not None or v_scale is not None:
        raise ValueError("rows of bf16 or fp32 have no scales")
    if block_table is not None and (block_table.dtype != torch.int32 or block_table.dim() != 2):
        raise ValueError("int32 block table [batch, max_blocks] expected")
    kv = dense_view(k, v) if block_table is None else paged_view(k, v, block_table)
    c = Cache(kv, dtype, k_scale.data_ptr() if k_scale is not None else None, v_scale.data_ptr() if v_scale is not None else None)
    c.tensors, c.index = tensors, k.get_device()
    c.lead = tuple(k.shape[:3]) if block_table is None else (k.shape[0], block_table.shape[0], k.shape[2])
    c.head_dim = k.shape[-1] * (2 if dtype == E2M1 else 1)
    return c


def make_rope(rot_dim: int, layout: int = ROPE_HALF, base: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0,
              original_len: int = 0, slow: float = 1.0, fast: float = 32.0, gain: float = 1.0) -> Rope:
    r = Rope()
    _check(lib().ams_rope_init(C.byref(r), layout, rot_dim, base, scaling, factor, original_len, slow, fast, gain), "ams_rope_init")
    return r


# The calls below run once per layer and token: their checks are written to cost the host little next to a launch (3 us).

def _cache_for(p: Params, c: Cache):
    """The GPU that the cache lies on, if it has the parameters' sizes."""
    if c.lead != (p.n_layers, p.batch, p.n_kv_heads) or c.head_dim != p.head_dim:
        raise ValueError(f"a cache of {c.lead} heads of {c.head_dim} channels does not fit the parameters")
    return c.index


def _load_args():
    """The compiled checks of tensor arguments (csrc/args.cpp) in the place of the two functions below, which the first use of either calls.  A module
    of this torch and Python: the entry points that do not use it do not need it."""
    global _arg, _token_rows
    try:
        from . import _args
    except ImportError as e:
        raise ImportError(f"{os.path.join(_HERE, '_args.so')} is missing or was built for another torch or Python: run "
                          "`python -m paper_2605_23200_amd.build` (or __graft_entry__.build())") from e
    _arg, _token_rows = _args.arg, _args.token_rows


def _arg(t: Optional[torch.Tensor], dtype: torch.dtype, numel: int, gpu: int, what: str):
    """Pointer of a contiguous tensor of at least `numel` elements on that GPU; None stays None."""
    _load_args()
    return _arg(t, dtype, numel, gpu, what)


def _token_rows(t: torch.Tensor, shape, dtype: torch.dtype, gpu: int, what: str):
    """(pointer, elements from token to token) of [L, B, n_new, heads, D]: any slice of a projection's output along the heads."""
    _load_args()
    return _token_rows(t, shape, dtype, gpu, what)


def _launch(fn, what: str, gpu: int, stream, *args):
    """Calls fn on the cache's GPU, whichever is current, and on that GPU's current stream unless one is given."""
    # (the raw handle of the current stream: making a Stream object of it costs as much as a launch)
    handle = torch._C._cuda_getCurrentRawStream(gpu) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == gpu:
        rc = fn(*args, handle)
    else:
        with torch.cuda.device(gpu):
            rc = fn(*args, handle)
    if rc != OK:
        raise AmsError(rc, what)


_ROWS = {F32: torch.float32, BF16: torch.bfloat16}


def ams_append(p, q, k, v, q_weight, k_weight, norm_eps, rope, positions, seq_lens, q_out, dst, lens_out=None, stream=None):
    """q [L, B, n_new, H * G, D] (or None, q_out too), k, v [L, B, n_new, H, D]; rope, the weights, positions and lens_out may be None."""
    gpu = _cache_for(p, dst)
    if k.dim() != 5:
        raise ValueError("k: [layers, batch, new, heads, channels] expected")
    (L, batch, H), D, n_new, rows, i32 = dst.lead, dst.head_dim, k.shape[2], _ROWS[p.kv_dtype], torch.int32
    HQ, kv_shape = H * p.group, (L, batch, n_new, H, D)
    qp, qs = _token_rows(q, (L, batch, n_new, HQ, D), rows, gpu, "q") if q is not None else (None, 0)
    kp, ks = _token_rows(k, kv_shape, rows, gpu, "k")
    vp, vs = _token_rows(v, kv_shape, rows, gpu, "v")
    x = NewTokens(qp, kp, vp, qs, ks, vs, _arg(q_weight, rows, D, gpu, "q_weight"), _arg(k_weight, rows, D, gpu, "k_weight"), norm_eps,
                  _arg(positions, i32, batch, gpu, "positions"), n_new)
    _launch((_lib or lib()).ams_append, "ams_append", gpu, stream, C.byref(p), C.byref(x), C.byref(rope) if rope is not None else None,
            _arg(seq_lens, i32, batch, gpu, "seq_lens"), _arg(q_out, rows, L * batch * HQ * n_new * D, gpu, "q_out"), C.byref(dst),
            _arg(lens_out, i32, batch, gpu, "lens_out"))


def ams_attend_workspace_bytes(p: Params) -> int:
    return int(lib().ams_attend_workspace_bytes(C.byref(p)))


def ams_attend(p, src, seq_lens, q, out, ws, lse=None, weights_in=None, weights_out=None, stream=None):
    gpu, rows, batch, D = _cache_for(p, src), _ROWS[p.kv_dtype], p.batch, p.head_dim
    units = p.n_layers * batch * p.n_kv_heads
    n, weights = units * p.group * p.window, units * p.t_stride
    _launch((_lib or lib()).ams_attend, "ams_attend", gpu, stream, C.byref(p), C.byref(src),
            _arg(seq_lens, torch.int32, batch, gpu, "seq_lens"), _arg(q, rows, n * D, gpu, "q"),
            _arg(out, rows, n * D, gpu, "out"), _arg(lse, torch.float32, n, gpu, "lse"),
            _arg(weights_in, torch.float32, weights, gpu, "weights_in"), _arg(weights_out, torch.float32, weights, gpu, "weights_out"),
            _arg(ws, torch.uint8, 0, gpu, "ws"), ws.numel())


def ams_recode(p, src, seq_lens, dst, idx=None, n_kept=None, credit_src=None, credit_dst=None, stream=None):
    gpu = _cache_for(p, src)
    if _cache_for(p, dst) != gpu:
        raise ValueError("both caches lie on one GPU")
    units = p.units
    kept = units * p.budget
    _launch((_lib or lib()).ams_recode, "ams_recode", gpu, stream, C.byref(p), C.byref(src),
            _arg(seq_lens, torch.int32, p.batch, gpu, "seq_lens"), _arg(idx, torch.int32, kept, gpu, "idx"),
            _arg(n_kept, torch.int32, units, gpu, "n_kept"), C.byref(dst),
            _arg(credit_src, torch.float32, units * p.t_stride, gpu, "credit_src") if credit_src is not None else None,
            _arg(credit_dst, torch.float32, kept, gpu, "credit_dst"))


def ams_evict_workspace_bytes(p: Params) -> int:
    return int(lib().ams_evict_workspace_bytes(C.byref(p)))


def ams_evict(p, src, seq_lens, weights, dst, weights_out, idx, n_kept, ws, lens_out=None, stream=None):
    gpu = _cache_for(p, src)
    if _cache_for(p, dst) != gpu:
        raise ValueError("both caches lie on one GPU")
    _launch((_lib or lib()).ams_evict, "ams_evict", gpu, stream, C.byref(p), C.byref(src),
            _arg(seq_lens, torch.int32, p.batch, gpu, "seq_lens"),
            _arg(weights, torch.float32, p.units * p.t_stride, gpu, "weights"), C.byref(dst),
            _arg(weights_out, torch.float32, p.units * p.t_stride, gpu, "weights_out"),
            _arg(idx, torch.int32, p.units * p.budget, gpu, "idx"), _arg(n_kept, torch.int32, p.units, gpu, "n_kept"),
            _arg(lens_out, torch.int32, p.batch, gpu, "lens_out"), _arg(ws, torch.uint8, 0, gpu, "ws"), ws.numel())


def ams_assign_pages(p, lens_from, lens_to, table, table_out, ring, state, state_out, starts=None, slots=None, lens_out=None, stream=None):
    """table, table_out int32 [batch, max_blocks] (may be one tensor), ring int32 [n_pages], state, state_out int32 [2], starts int32
    [batch + 1], slots int64, any length."""
    gpu, i32 = table.get_device(), torch.int32
    if gpu < 0 or table.dim() != 2 or table.shape[0] != p.batch or table_out.shape != table.shape or ring.dim() != 1:
        raise ValueError(f"block tables [{p.batch}, max_blocks] on a GPU and a ring of one dimension expected")
    n = table.numel()
    x = Pages(_arg(table, i32, n, gpu, "table"), _arg(table_out, i32, n, gpu, "table_out"), table.shape[1], ring.numel(),
              _arg(ring, i32, 1, gpu, "ring"), _arg(state, i32, 2, gpu, "state"), _arg(state_out, i32, 2, gpu, "state_out"))
    _launch((_lib or lib()).ams_assign_pages, "ams_assign_pages", gpu, stream, C.byref(p), C.byref(x),
            _arg(lens_from, i32, p.batch, gpu, "lens_from"), _arg(lens_to, i32, p.batch, gpu, "lens_to"),
            _arg(lens_out, i32, p.batch, gpu, "lens_out"), _arg(starts, i32, p.batch + 1, gpu, "starts"),
            _arg(slots, torch.int64, 0, gpu, "slots"), slots.numel() if slots is not None else 0)


@dataclass
class StepIntermediates:
    u: torch.Tensor
    g: torch.Tensor
    m_used: torch.Tensor
    bounds: torch.Tensor
    seg_mass: torch.Tensor
    quota: torch.Tensor


def workspace_tensors(p: Params, ws: torch.Tensor) -> StepIntermediates:
    """Typed views of the intermediates ams_compress_step left in `ws` (a uint8 device tensor)."""
    lay = ams_workspace_layout(p)
    U, S, ts = p.units, p.n_segments, p.t_stride

    def view(off, n, dtype, shape):
        return ws[off:off + n * 4].view(dtype).view(*shape)

    return StepIntermediates(
        u=view(lay.u, U * ts, torch.float32, (U, ts)), g=view(lay.g, U * ts, torch.float32, (U, ts)),
        m_used=view(lay.m_used, U * ts, torch.float32, (U, ts)),
        bounds=view(lay.bounds, U * (S + 1), torch.int32, (U, S + 1)),
        seg_mass=view(lay.seg_mass, U * S, torch.float32, (U, S)),
        quota=view(lay.quota, U * S, torch.int32, (U, S)))
