"""The operators around a bounded cache, as they are measured: what each computes in plain torch, and the library's calls.

A serving loop writes new tokens into a cache (`ams_append`), attends to it (`ams_attend`), takes rows to and from 8 bits
(`ams_recode`) and evicts by accumulated attention weight (`ams_evict`).  A cache in 8 bits holds one-byte codes and, for
every block of 16 positions of a (layer, sequence, KV head), one scale for the keys and one for the values: a power of two,
the least that takes the block's largest magnitude to 127 (int8) or 448 (e4m3) or less.

A case is a dict:
  kind      "append" | "attend" | "recode" | "evict"
  layers, batch, heads, group, dim, dtype ("bf16" | "f32")
  code      "e4m3" | "int8" | "plain": what the cache holds ("append": the cache written; "recode": what rows are packed to)
  length, shortest   cache lengths are spread over [shortest, length] (equal: all sequences have that length)
  paged     pages of 16 positions and a block table; else one slab per (layer, sequence, KV head)
  append:   new (tokens per sequence), layout ("half" | "interleaved"), rotated (channels), scaling ("none" | "linear" |
            "base" | "parts"), factor, norm, first (positions begin there: a bounded cache is shorter than its context)
  attend:   window (queries per head), causal, weights (accumulate them)
  recode:   keep (rows gathered per unit; 0: the whole cache to 8 bits and back)
  evict:    budget, sink, last

Codes of e4m3 come back as the floating type that they are, with their scales; int8 is read back into rows first.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
BLOCK = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
MOST = {"e4m3": 448.0, "int8": 127.0}
EPS = 1e-6
BASE = 500000.0
ORIGINAL = 8192
SLOW, FAST = 1.0, 32.0


def _case(name, kind, **kw):
    c = dict(kind=kind, layers=1, batch=1, heads=8, group=4, dim=128, dtype="bf16", code="e4m3", length=4096, shortest=0,
             paged=False)
    c.update({"append": dict(new=1, layout="half", rotated=128, scaling="none", factor=1.0, norm=True, first=0),
              "attend": dict(window=1, causal=False, weights=True), "recode": dict(keep=0),
              "evict": dict(budget=2048, sink=4, last=32)}[kind])
    c.update(kw)
    c["shortest"] = c["shortest"] or c["length"]
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one sequence's next token in one layer, into the bf16 cache that a compression event reads
        _case("append-one", "append", code="plain", length=2305),
        # the next token of 64 sequences, into an 8-bit paged cache; half of the channels rotate, far positions
        _case("append-batch", "append", batch=64, length=4096, shortest=700, paged=True, layout="interleaved", rotated=64,
              scaling="parts", factor=32.0, first=200000),
        # a piece of four prompts
        _case("append-prompt", "append", batch=4, length=1111, shortest=640, new=509, scaling="linear", factor=4.0),
        # one token over one bounded cache: latency
        _case("attend-one", "attend", code="int8", length=2177),
        # the next token of 64 sequences of 4096 to 16384 positions in pages
        _case("attend-batch", "attend", batch=64, length=16384, shortest=4096, paged=True),
        # one token over a long cache
        _case("attend-long", "attend", heads=4, group=7, code="int8", length=131072),
        # 32 tokens at once, causal (a draft verified, a window replayed)
        _case("attend-window", "attend", code="int8", length=32768, window=32, causal=True),
        # fp32 queries, 64 channels, several layers at once
        _case("attend-f32-d64", "attend", layers=6, batch=4, heads=2, group=7, dim=64, dtype="f32", window=2, length=9001,
              shortest=700, causal=True),
        # what a compression event over all layers keeps, into an 8-bit cache
        _case("recode-event", "recode", layers=32, length=32768, keep=2048),
        # a ragged batch of prompts to 8 bits and read back
        _case("recode-whole", "recode", layers=2, batch=8, length=8001, shortest=1500, code="int8"),
        # all layers of one sequence back to the budget, as between two events
        _case("evict-short", "evict", layers=32, length=2176),
        # long caches of a ragged batch in pages
        _case("evict-long", "evict", layers=4, batch=6, heads=4, group=7, length=131072, shortest=40000, budget=4096, paged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attend", "attend", "recode", "evict"))
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    code = rng.choice(("e4m3", "int8"))
    heads, group = rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 2, 4, 4, 7, 8))
    dim = rng.choice((64, 128, 128, 128))
    paged = rng.random() < 0.4
    length = _log(rng, 300, 131072) if kind != "append" else _log(rng, 300, 8192)
    most = (1 << 29) // (length * heads * dim)  # (layer, sequence) pairs: a quarter of the largest listed cache
    if kind == "append":
        most = min(most, 64)
    pairs = max(1, min(_log(rng, 1, 128), most))
    batch = max(1, min(pairs, rng.choice((1, 1, 2, 4, 8, 16, 64))))
    shortest = length if batch == 1 or rng.random() < 0.3 else max(200, int(length * rng.uniform(0.1, 0.9)))
    kw = dict(layers=max(1, pairs // batch) if kind != "append" else 1, batch=batch, heads=heads, group=group, dim=dim,
              dtype=dtype, code=code, length=length, shortest=shortest, paged=paged)
    if kind == "append":
        new = 1 if rng.random() < 0.5 else min(_log(rng, 2, 512), 4096 // batch, shortest // 2)
        kw.update(new=max(1, new), code=rng.choice(("e4m3", "plain")), layout=rng.choice(("half", "interleaved")),
                  rotated=rng.choice((dim, dim, dim // 2, 2 * rng.randint(2, dim // 2))), norm=rng.random() < 0.7,
                  scaling=rng.choice(("none", "linear", "base", "parts")), factor=rng.choice((2.0, 8.0, 32.0)),
                  first=rng.choice((0, 0, rng.randint(1, 1000000))))
    elif kind == "attend":
        window = 1 if rng.random() < 0.6 else rng.randint(2, 32)
        if length * batch * kw["layers"] * heads * group * window > 1 << 27:  # the plain form keeps every probability
            window = 1
        kw.update(window=window, causal=rng.random() < 0.7, weights=rng.random() < 0.7)
    elif kind == "recode":
        kw.update(keep=0 if rng.random() < 0.4 else max(1, int(shortest / rng.choice((1.05, 2, 8, 16)))))
    else:
        budget = max(64, int(shortest / rng.choice((1.05, 2, 8, 16, 32))))
        kw.update(budget=min(budget, shortest), sink=rng.choice((0, 4, 16)), last=rng.choice((0, 32, 33)))
    return _case("", kind, **kw)


# ---------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Cache lengths of the batch: a property of the case, spread over [shortest, length], the longest among them."""
    r = random.Random(case["length"] * 31 + case["batch"])
    lens = [case["length"]] + [r.randint(case["shortest"], case["length"]) for _ in range(case["batch"] - 1)]
    r.shuffle(lens)
    return lens


def _blocks(n):
    return -(-n // BLOCK)


def _units(case):
    return case["layers"] * case["batch"] * case["heads"]


def _table(case, lens, seed):
    """Block table over a shuffled pool that holds just these sequences; entries past a sequence's end are -1."""
    counts = [_blocks(n) for n in lens]
    perm = torch.randperm(sum(counts), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lens), max(counts)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = perm[at:at + n]
        at += n
    return table.to(DEVICE), at


def _to_pool(x, table, n_blocks, fill):
    """[B, H, blocks * 16 or blocks, ...] of one layer into a pool [n_blocks * 16 or n_blocks, H, ...]."""
    per = x.shape[2] // table.shape[1]
    pool = torch.full((n_blocks, per, x.shape[1]) + x.shape[3:], fill, dtype=torch.float32, device=DEVICE).to(x.dtype)
    b, j = (table >= 0).nonzero(as_tuple=True)
    rows = x.reshape(x.shape[0], x.shape[1], table.shape[1], per, *x.shape[3:]).transpose(1, 2)[b, j]
    pool[table[b, j].long()] = rows.transpose(1, 2)
    return pool.reshape(n_blocks * per, x.shape[1], *x.shape[3:])


def _rows(gen, case, T):
    """Rows of one layer [B, H, T, D], float32: a few loud channels, and tokens of different loudness."""
    shape = (case["batch"], case["heads"], T, case["dim"])
    channel = 1 + 3 * (torch.rand((1, case["heads"], 1, case["dim"]), device=DEVICE, generator=gen) > 0.96)
    token = torch.randn((case["batch"], 1, T, 1), device=DEVICE, generator=gen).mul_(0.3).exp_()
    return torch.randn(shape, device=DEVICE, generator=gen).mul_(channel).mul_(token)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    L, N_B, H, G, D = (case[k] for k in ("layers", "batch", "heads", "group", "dim"))
    kind, dtype, code = case["kind"], DTYPES[case["dtype"]], case["code"]
    lens = _lengths(case)
    s = {"case": case, "lens": torch.tensor(lens, dtype=torch.int32, device=DEVICE), "handle": None}
    new = case.get("new", 0)
    table, n_blocks = _table(case, [n + new for n in lens], seed) if case["paged"] else (None, 0)
    s["table"] = table
    T = max(lens) + new
    padded = _blocks(T) * BLOCK if kind != "recode" else T
    plain_source = kind == "recode" or (kind == "append" and code == "plain")
    inside = (torch.arange(_blocks(T) * BLOCK, device=DEVICE) < s["lens"][:, None])[:, None, :, None]  # [B, 1, rows, 1]
    for name in ("k", "v"):
        rows, scales = [], []
        for _ in range(L):
            x = _rows(gen, case, padded if not case["paged"] else _blocks(T) * BLOCK)
            if name == "k" and kind == "attend":  # some stretches are what the recent queries look at
                x[:, :, ::37] *= 1.5
            if plain_source:
                x = x.to(dtype)
                rows.append(_to_pool(x, table, n_blocks, 0.0) if case["paged"] else x)
                continue
            codes, scale = _pack(torch.where(inside, x, torch.zeros((), device=DEVICE)), code)
            rows.append(_to_pool(codes, table, n_blocks, 0.0) if case["paged"] else codes)
            scales.append(_to_pool(scale, table, n_blocks, 0.0) if case["paged"] else scale)
        s[name] = torch.stack(rows)
        if scales:
            s[name + "_scale"] = torch.stack(scales)
        del rows, scales
    if kind == "append":
        qkv = torch.randn((L, N_B, new, (G + 2) * H, D), device=DEVICE, generator=gen).to(dtype)  # one projection's output
        s["new_q"], s["new_k"], s["new_v"] = qkv[..., :G * H, :], qkv[..., G * H:(G + 1) * H, :], qkv[..., (G + 1) * H:, :]
        for name in ("q_weight", "k_weight"):
            s[name] = (1 + 0.2 * torch.randn(D, device=DEVICE, generator=gen)).to(dtype) if case["norm"] else None
        s["first"] = s["lens"] + case["first"]
        s["q_out"] = torch.zeros((L, N_B, H * G, new, D), dtype=dtype, device=DEVICE)
        s["lens_out"] = torch.zeros_like(s["lens"])
    elif kind == "attend":
        W = case["window"]
        s["q"] = torch.randn((L, N_B, H * G, W, D), device=DEVICE, generator=gen).to(dtype)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((L, N_B, H * G, W), device=DEVICE)
        if case["weights"]:
            s["weights"] = torch.rand((_units(case), T), device=DEVICE, generator=gen).pow_(4) * 3
            s["weights_out"] = torch.zeros_like(s["weights"])
    elif kind == "recode":
        keep = case["keep"]
        if keep:
            order = torch.rand((_units(case), T), device=DEVICE, generator=gen)
            order.masked_fill_(~inside[:, 0, :T, 0].repeat_interleave(H, 0).repeat(L, 1), 2.0)
            s["idx"] = order.argsort(1)[:, :keep].sort(1).values.to(torch.int32).contiguous()
            s["n_kept"] = torch.full((_units(case),), keep, dtype=torch.int32, device=DEVICE)
        s.update(_fresh(case, keep or T, code))
        if not keep or code == "int8":
            s["back_k"] = torch.zeros((L, N_B, H, keep or T, D), dtype=dtype, device=DEVICE)
            s["back_v"] = torch.zeros_like(s["back_k"])
    else:
        weights = torch.randn((_units(case), T), device=DEVICE, generator=gen).mul_(1.5).exp_()
        s["weights"], s["weights_out"] = weights, torch.zeros_like(weights)
        s["idx"] = torch.full((_units(case), case["budget"]), -1, dtype=torch.int32, device=DEVICE)
        s["n_kept"] = torch.zeros(_units(case), dtype=torch.int32, device=DEVICE)
        s.update(_fresh(case, case["budget"], code))
        if code == "int8":
            s["back_k"] = torch.zeros((L, N_B, H, case["budget"], D), dtype=torch.bfloat16, device=DEVICE)
            s["back_v"] = torch.zeros_like(s["back_k"])
    return s


def _fresh(case, rows, code):
    """An empty 8-bit slab of that many rows per unit."""
    shape = (case["layers"], case["batch"], case["heads"], rows, case["dim"])
    out = {}
    for name in ("k", "v"):
        out["to_" + name] = torch.zeros(shape, dtype=CODES[code], device=DEVICE)
        out["to_" + name + "_scale"] = torch.zeros(shape[:3] + (_blocks(rows),), device=DEVICE)
    return out


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _own(s)
    return {"append": _append, "attend": _attend, "recode": _recode, "evict": _evict}[s["case"]["kind"]](s)


def _own(s):
    from paper_2605_23200_amd import binding as B
    case, kind = s["case"], s["case"]["kind"]
    if s["handle"] is None:
        s["handle"] = _handle(B, s)
    h = s["handle"]
    if kind == "append":
        B.ams_append(h["p"], s["new_q"], s["new_k"], s["new_v"], s["q_weight"], s["k_weight"], EPS, h["rope"], s["first"],
                     s["lens"], s["q_out"], h["cache"], s["lens_out"])
        return _appended(s, s["q_out"], s["lens_out"])
    if kind == "attend":
        B.ams_attend(h["p"], h["cache"], s["lens"], s["q"], s["out"], h["ws"], s["lse"], s.get("weights"), s.get("weights_out"))
        return {k: s[k] for k in ("out", "lse", "weights_out") if k in s}
    if kind == "recode":
        if case["keep"]:
            B.ams_recode(h["p"], h["cache"], None, h["to"], s["idx"], s["n_kept"])
        else:
            B.ams_recode(h["p"], h["cache"], s["lens"], h["to"])
        if "back" in h:
            B.ams_recode(h["p_back"], h["to"], h["kept"] if case["keep"] else s["lens"], h["back"])
        return _recoded(s)
    B.ams_evict(h["p"], h["cache"], s["lens"], s["weights"], h["to"], s["weights_out"], s["idx"], s["n_kept"], h["ws"],
                h["kept"])
    if "back" in h:
        B.ams_recode(h["p_back"], h["to"], h["kept"], h["back"])
    return dict(_recoded(s), idx=s["idx"], n_kept=s["n_kept"], weights=s["weights_out"])


def _handle(B, s):
    """What a user's program keeps from call to call: parameters, views, the rotation's table, the workspace."""
    case, kind = s["case"], s["case"]["kind"]
    T = s["case"]["length"] + case.get("new", 0)
    kept = case.get("keep") or case.get("budget") or T
    common = dict(n_layers=case["layers"], batch=case["batch"], n_kv_heads=case["heads"], group=case["group"],
                  window=case.get("window", 1), head_dim=case["dim"], kv_dtype=B.F32 if case["dtype"] == "f32" else B.BF16,
                  n_segments=1)
    h = {"p": B.make_params(t_max=T, budget=kept, causal=case.get("causal", False), n_sink=case.get("sink", 0),
                            n_last=case.get("last", 0), **common)}
    h["cache"] = B.cache_view(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"), block_table=s["table"])
    if kind == "append":
        kinds = {"none": B.ROPE_PLAIN, "linear": B.ROPE_LINEAR, "base": B.ROPE_BASE, "parts": B.ROPE_BY_PARTS}
        h["rope"] = B.make_rope(case["rotated"], layout=B.ROPE_HALF if case["layout"] == "half" else B.ROPE_INTERLEAVED,
                                base=BASE, scaling=kinds[case["scaling"]], factor=case["factor"], original_len=ORIGINAL,
                                slow=SLOW, fast=FAST, gain=_gain(case))
    if kind == "attend":
        h["ws"] = torch.empty(B.ams_attend_workspace_bytes(h["p"]), dtype=torch.uint8, device=DEVICE)
    if kind == "evict":
        h["ws"] = torch.empty(B.ams_evict_workspace_bytes(h["p"]), dtype=torch.uint8, device=DEVICE)
    if kind in ("recode", "evict"):
        # rows per sequence of what is written: what a gather is asked for; an eviction says it anew every time
        h["kept"] = torch.full((case["batch"],), kept, dtype=torch.int32, device=DEVICE)
        h["to"] = B.cache_view(s["to_k"], s["to_v"], s["to_k_scale"], s["to_v_scale"])
        if "back_k" in s:
            h["back"] = B.cache_view(s["back_k"], s["back_v"])
            back = dict(common, kv_dtype=B.F32 if s["back_k"].dtype == torch.float32 else B.BF16)
            h["p_back"] = B.make_params(t_max=kept, budget=kept, **back)
    return h


def _appended(s, q, lens):
    out = {"q": q, "lens": lens, "k": s["k"], "v": s["v"]}
    return dict(out, k_scale=s["k_scale"], v_scale=s["v_scale"]) if "k_scale" in s else out


def _recoded(s):
    """The rows written: as e4m3 values and their scales, or read back."""
    if "back_k" in s:
        return {"k": s["back_k"], "v": s["back_v"]}
    return {k: s["to_" + k] for k in ("k", "v", "k_scale", "v_scale")}


# ---- the plain forms ----

def _pack(x, code):
    """Rows [..., T, D] in float32 -> codes [..., T, D] and scales [..., ceil(T / 16)]."""
    T = x.shape[-2]
    x = torch.nn.functional.pad(x, (0, 0, 0, -T % BLOCK)).unflatten(-2, (-1, BLOCK))
    scale = _scale(x.abs().amax((-1, -2)), MOST[code])
    y = (x / torch.where(scale > 0, scale, torch.ones_like(scale))[..., None, None]).flatten(-3, -2)[..., :T, :]
    return (y.round() if code == "int8" else y).to(CODES[code]), scale


def _scale(largest, most):
    """The least power of two (from 2^-120 on) that takes `largest` to `most` or less; 0 for 0."""
    m, e = torch.frexp(largest)
    m0, e0 = math.frexp(most)
    power = (e - e0 + (m > m0)).clamp(min=-120)
    return torch.where(largest > 0, torch.ldexp(torch.ones_like(largest), power), torch.zeros_like(largest))


def _from_pool(x, table):
    """A pool [L, n_blocks * per, H, ...] through its table: [L, B, H, blocks * per, ...]."""
    per = BLOCK if x.dim() == 4 else 1
    x = x.unflatten(1, (-1, per))[:, table.long().clamp(min=0)]   # [L, B, blocks, per, H, ...]
    return x.movedim(4, 2).flatten(3, 4)


def _values(s, name):
    """A cache's rows [L, B, H, T, D] in float32."""
    x = s[name] if s["table"] is None else _from_pool(s[name], s["table"])
    if name + "_scale" not in s:
        return x.float()
    scale = s[name + "_scale"] if s["table"] is None else _from_pool(s[name + "_scale"], s["table"])
    return x.float().mul_(scale.repeat_interleave(BLOCK, -1)[..., :x.shape[3], None])


def _gain(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "parts" else 1.0


def _frequencies(case):
    """Radians per position of every rotated pair, float64."""
    n = case["rotated"]
    i = torch.arange(0, n, 2, dtype=torch.float64, device=DEVICE)
    base = BASE * case["factor"] ** (n / (n - 2)) if case["scaling"] == "base" else BASE
    f = base ** (-i / n)
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "parts":
        turns = f * (ORIGINAL / (2 * math.pi))
        keep = ((turns - SLOW) / (FAST - SLOW)).clamp(0, 1)
        f = f * (keep + (1 - keep) / case["factor"])
    return f


def _normed(x, weight):
    x = x.float()
    if weight is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _turned(x, cos, sin, case):
    """x [L, B, W, heads, D]; cos, sin [B, W, 1, rotated / 2]."""
    n = case["rotated"]
    if case["layout"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., n:]], -1)


def _append(s):
    case, new = s["case"], s["case"]["new"]
    pos = s["first"].double()[:, None] + torch.arange(new, device=DEVICE)
    angle = pos[..., None, None] * _frequencies(case)
    cos, sin = (angle.cos() * _gain(case)).float(), (angle.sin() * _gain(case)).float()
    q = _turned(_normed(s["new_q"], s["q_weight"]), cos, sin, case).to(s["q_out"].dtype).movedim(3, 2).contiguous()
    k = _turned(_normed(s["new_k"], s["k_weight"]), cos, sin, case)
    at = s["lens"].long()[:, None] + torch.arange(new, device=DEVICE)      # [B, W] rows written
    b = torch.arange(case["batch"], device=DEVICE)[:, None]
    for name, x in (("k", k), ("v", s["new_v"].float())):
        if case["code"] == "plain":
            if s["table"] is None:
                s[name][:, b, :, at] = x.to(s[name].dtype).movedim(0, 2)
            else:
                s[name][:, s["table"].long()[b, at // BLOCK] * BLOCK + at % BLOCK] = x.to(s[name].dtype)
            continue
        _append_packed(s, name, x, at, b)
    return _appended(s, q, s["lens"] + new)


def _append_packed(s, name, x, at, b):
    """The touched blocks: the rows that were there under the new scale, the new rows beside them."""
    case = s["case"]
    most, codes, scales = MOST[case["code"]], s[name], s[name + "_scale"]
    first = s["lens"].long() // BLOCK
    n = (case["new"] + 2 * BLOCK - 2) // BLOCK
    block = first[:, None] + torch.arange(n, device=DEVICE)                 # [B, n]
    touched = block * BLOCK < s["lens"][:, None] + case["new"]
    block = torch.where(touched, block, first[:, None])                     # a block past the end: the first once more
    if s["table"] is None:
        old = codes.unflatten(3, (-1, BLOCK))[:, b, :, block].movedim(2, 0)  # [L, B, n, H, 16, D]
        old_scale = scales[:, b, :, block].movedim(2, 0)                     # [L, B, n, H]
    else:
        page = s["table"].long()[b, block]
        old = codes.unflatten(1, (-1, BLOCK))[:, page].movedim(4, 3)
        old_scale = scales[:, page]
    row = block[..., None] * BLOCK + torch.arange(BLOCK, device=DEVICE)      # [B, n, 16]
    age = row - s["lens"][:, None, None]                                     # < 0: was there
    fresh = x[:, b[..., None], age.clamp(0, case["new"] - 1)].movedim(4, 3)  # [L, B, n, H, 16, D]
    is_new = ((age >= 0) & (age < case["new"]))[:, :, None, :, None]
    was = (age < 0)[:, :, None, :, None]
    need = _scale((fresh * is_new).abs().amax((-1, -2)), most)
    had = torch.where((age[..., 0] < 0)[:, :, None], old_scale, torch.zeros_like(need))
    scale = torch.maximum(need, had)
    div = torch.where(scale > 0, scale, torch.ones_like(scale))[..., None, None]
    y = torch.where(was, old.float() * (had[..., None, None] / div), fresh / div)
    y = (y.round() if case["code"] == "int8" else y).to(codes.dtype)
    y = torch.where(is_new | was, y.view(torch.int8), old.contiguous().view(torch.int8)).view(codes.dtype)
    if s["table"] is None:
        codes.unflatten(3, (-1, BLOCK))[:, b, :, block] = y.movedim(0, 2)
        scales[:, b, :, block] = scale.movedim(0, 2)
    else:
        codes.unflatten(1, (-1, BLOCK))[:, page] = y.movedim(3, 4)
        scales[:, page] = scale


def _attend(s):
    case = s["case"]
    L, N_B, H, G, W, D = (case[k] for k in ("layers", "batch", "heads", "group", "window", "dim"))
    k, v = _values(s, "k"), _values(s, "v")
    T = k.shape[3]
    q = s["q"].float().reshape(L * N_B * H, G * W, D)
    x = torch.matmul(q, k.reshape(-1, T, D).transpose(1, 2)).mul_(1 / math.sqrt(D)).reshape(L, N_B, H, G, W, T)
    limit = s["lens"].long()[:, None] - (torch.arange(W - 1, -1, -1, device=DEVICE) if case["causal"] else 0)  # [B, W]
    seen = (torch.arange(T, device=DEVICE) < limit[..., None]).reshape(N_B, 1, 1, -1, T)
    x = torch.where(seen, x, torch.full((), -math.inf, device=DEVICE))
    largest = x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = x.sub_(largest).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total.clamp(min=1e-30))
    out = torch.matmul(p.reshape(-1, G * W, T), v.reshape(-1, T, D)).reshape(L, N_B, H * G, W, D).to(s["q"].dtype)
    lse = (largest + total.log()).reshape(L, N_B, H * G, W)
    if not case["weights"]:
        return {"out": out, "lse": lse}
    more = p.sum((3, 4)).reshape(-1, T)[:, :s["weights"].shape[1]]
    inside = (torch.arange(more.shape[1], device=DEVICE) < s["lens"][:, None]).repeat_interleave(H, 0).repeat(L, 1)
    return {"out": out, "lse": lse, "weights_out": torch.where(inside, s["weights"] + more, s["weights_out"])}


def _picked(s, name, idx):
    """Rows idx [units, n] of a cache, [L, B, H, n, D], in float32."""
    case = s["case"]
    L, N_B, H = case["layers"], case["batch"], case["heads"]
    t = idx.long().reshape(L, N_B, H, -1)
    l, b, h = (torch.arange(n, device=DEVICE).reshape(shape) for n, shape in
               ((L, (-1, 1, 1, 1)), (N_B, (1, -1, 1, 1)), (H, (1, 1, -1, 1))))
    scale = s.get(name + "_scale")
    if s["table"] is None:
        x = s[name][l, b, h, t].float()
        return x if scale is None else x.mul_(scale[l, b, h, t // BLOCK][..., None])
    page = s["table"].long()[b, t // BLOCK]
    x = s[name][l, page * BLOCK + t % BLOCK, h].float()
    return x if scale is None else x.mul_(scale[l, page, h][..., None])


def _recode(s):
    case = s["case"]
    out = {}
    for name in ("k", "v"):
        if case["keep"]:
            x = _picked(s, name, s["idx"])
        else:
            x = _values(s, name)[:, :, :, :case["length"]]
            x = torch.where((torch.arange(x.shape[3], device=DEVICE) < s["lens"][:, None])[:, None, :, None], x, 0.0)
        out[name], out[name + "_scale"] = _pack(x, case["code"])
    return _as_rows(s, out)


def _as_rows(s, out):
    if "back_k" not in s:
        return out
    return {name: (out[name].float() * out[name + "_scale"].repeat_interleave(BLOCK, -1)[..., :out[name].shape[3], None])
            .to(s["back_k"].dtype) for name in ("k", "v")}


def _evict(s):
    case, w = s["case"], s["weights"]
    keep, H, L = case["budget"], case["heads"], case["layers"]
    lens = s["lens"].repeat_interleave(H).repeat(L)[:, None]
    t = torch.arange(w.shape[1], device=DEVICE)
    sinks = min(case["sink"], keep)
    always = (t < sinks) | (t >= lens - min(case["last"], keep - sinks))
    rank = torch.where(t < lens, torch.where(always, math.inf, w), -math.inf)
    idx = rank.sort(dim=1, descending=True, stable=True).indices[:, :keep].sort(1).values
    out = {}
    for name in ("k", "v"):
        out[name], out[name + "_scale"] = _pack(_picked(s, name, idx), case["code"])
    carried = torch.zeros_like(w)
    carried[:, :keep] = w.gather(1, idx)
    n_kept = torch.full((w.shape[0],), keep, dtype=torch.int32, device=DEVICE)
    return dict(_as_rows(s, out), idx=idx.to(torch.int32), n_kept=n_kept, weights=carried)


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    L, N_B, H, G, D = (case[k] for k in ("layers", "batch", "heads", "group", "dim"))
    tokens = L * H * sum(_lengths(case))                        # rows of K, and of V
    row, scale = D, 4 / BLOCK                                   # of a row in 8 bits
    if case["kind"] == "append":
        new = L * N_B * case["new"]
        read = new * (G + 2) * H * D * e
        written = new * (G * H * D * e + 2 * H * (D * e if case["code"] == "plain" else row + scale))
        return {"bytes": read + written, "flops": new * (G + 1) * H * D * 8}
    if case["kind"] == "attend":
        n = G * case["window"]
        rows = L * N_B * H * n
        total = tokens * (2 * (row + scale) + (8 if case["weights"] else 0)) + rows * (2 * D * e + 4)
        return {"bytes": total, "flops": 4 * tokens * n * D}
    if case["kind"] == "recode":
        moved = L * N_B * H * case["keep"] or tokens
        back = D * e if case["code"] == "int8" or not case["keep"] else 0
        return {"bytes": moved * 2 * (D * e + row + scale + (row + scale if back else 0) + back), "flops": moved * 2 * D * 4}
    kept = L * N_B * H * case["budget"]
    back = kept * 2 * (row + scale + 2 * D) if case["code"] == "int8" else 0
    return {"bytes": tokens * 4 + kept * (4 * (row + scale) + 12) + back, "flops": tokens + kept * 4 * D}


# ---------------------------------------------------------------------------------------------------------------
# The same outputs in 64 bits, unit by unit
# ---------------------------------------------------------------------------------------------------------------

def _exact_scale(block, most):
    """The block's scale, as a float64 tensor of one value per leading index, by trying powers."""
    largest = block.abs().amax((-1, -2))
    power = torch.floor(torch.log2(largest.clamp(min=1e-300) / most)) - 1
    for _ in range(3):
        power = torch.where(largest > most * torch.exp2(power), power + 1, power)
    return torch.where(largest > 0, torch.exp2(power.clamp(min=-120)), torch.zeros_like(largest))


def _exact_round(y, code):
    """To the nearest code's value, ties to the even one."""
    if code == "int8":
        return torch.round(y)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)   # normal numbers from 2^-6 on
    return torch.round(y / step) * step


def _exact_pack(x, code):
    """x [units, T, D] float64 -> values of the codes, scales."""
    units, T, D = x.shape
    full = torch.zeros((units, _blocks(T) * BLOCK, D), dtype=torch.float64, device=DEVICE)
    full[:, :T] = x
    full = full.reshape(units, -1, BLOCK, D)
    scale = _exact_scale(full, MOST[code])
    y = torch.where(scale[..., None, None] > 0, full / scale.clamp(min=2.0 ** -130)[..., None, None], 0.0)
    return _exact_round(y, code).reshape(units, -1, D)[:, :T], scale


def _slab(s, name, l, b, h, T):
    """Rows 0 .. T of one unit, float64."""
    t = torch.arange(T, device=DEVICE)
    scale = s.get(name + "_scale")
    if s["table"] is None:
        x = s[name][l, b, h, :T].double()
        return x if scale is None else x * scale[l, b, h, t // BLOCK].double()[:, None]
    page = s["table"][b].long()[t // BLOCK]
    x = s[name][l, page * BLOCK + t % BLOCK, h].double()
    return x if scale is None else x * scale[l, page, h].double()[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "recode": _exact_recode, "evict": _exact_evict}[case["kind"]](s)


def _exact_append(s):
    case = s["case"]
    N_B, H, G, D, new, n = (case[k] for k in ("batch", "heads", "group", "dim", "new", "rotated"))
    first, second = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
    f = [BASE ** (-2 * i / n) for i in range(n // 2)]
    if case["scaling"] == "base":
        f = [(BASE * case["factor"] ** (n / (n - 2))) ** (-2 * i / n) for i in range(n // 2)]
    if case["scaling"] == "linear":
        f = [x / case["factor"] for x in f]
    if case["scaling"] == "parts":
        mix = [min(1.0, max(0.0, (x * ORIGINAL / 2 / math.pi - SLOW) / (FAST - SLOW))) for x in f]
        f = [x * m + x / case["factor"] * (1 - m) for x, m in zip(f, mix)]
    f = torch.tensor(f, dtype=torch.float64, device=DEVICE)
    q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEVICE)
    packed = case["code"] != "plain"
    out = {"lens": None}
    for name in ("k", "v"):
        out[name] = s[name].double()
        if packed:
            out[name + "_scale"] = s[name + "_scale"].double()
    for b in range(N_B):
        had = int(s["lens"][b])
        z = torch.polar(torch.full((new, n // 2), _gain(case), dtype=torch.float64, device=DEVICE),
                        (int(s["first"][b]) + torch.arange(new, device=DEVICE, dtype=torch.float64))[:, None] * f)
        rows = {"v": s["new_v"][0, b].double()}
        for name, x, weight in (("q", s["new_q"], s["q_weight"]), ("k", s["new_k"], s["k_weight"])):
            x = x[0, b].double()                                   # [new, heads, D]
            if weight is not None:
                x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.double()
            y = x.clone()
            turned = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z[:, None]
            y[..., first], y[..., second] = turned.real, turned.imag
            rows[name] = y
        q[0, b] = rows["q"].transpose(0, 1)
        for name in ("k", "v"):
            x = rows[name].transpose(0, 1)                         # [H, new, D]
            t = torch.arange(had, had + new, device=DEVICE)
            if s["table"] is not None:
                place = s["table"][b].long()[t // BLOCK] * BLOCK + t % BLOCK
            if not packed:
                if s["table"] is None:
                    out[name][0, b, :, had:had + new] = x
                else:
                    out[name][0, place] = x.transpose(0, 1)
                continue
            for j in range(had // BLOCK, _blocks(had + new)):
                lo, hi = max(had, j * BLOCK), min(had + new, (j + 1) * BLOCK)
                old = lo - j * BLOCK
                mine = x[:, lo - had:hi - had]
                scale = _exact_scale(mine, MOST[case["code"]])
                if s["table"] is None:
                    codes, scales = out[name][0, b, :, j * BLOCK:(j + 1) * BLOCK], out[name + "_scale"][0, b, :, j]
                else:
                    page = int(s["table"][b, j])
                    codes = out[name][0, page * BLOCK:(page + 1) * BLOCK].transpose(0, 1)
                    scales = out[name + "_scale"][0, page]
                if old:
                    scale = torch.maximum(scale, scales)
                    ratio = torch.where(scale > 0, scales / scale.clamp(min=2.0 ** -130), 0.0)[:, None, None]
                    codes[:, :old] = _exact_round(codes[:, :old] * ratio, case["code"])
                safe = scale.clamp(min=2.0 ** -130)[:, None, None]
                codes[:, old:old + hi - lo] = torch.where(scale[:, None, None] > 0, _exact_round(mine / safe, case["code"]), 0.0)
                scales.copy_(scale)
    return dict(out, q=q)


def _exact_attend(s):
    case = s["case"]
    L, N_B, H, G, W, D = (case[k] for k in ("layers", "batch", "heads", "group", "window", "dim"))
    lens = s["lens"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEVICE)
    weights = s["weights_out"].double() if case["weights"] else None
    for unit in range(L * N_B * H):
        l, b, h = unit // (N_B * H), unit // H % N_B, unit % H
        T = lens[b]
        k, v = _slab(s, "k", l, b, h, T), _slab(s, "v", l, b, h, T)
        q = s["q"][l, b, h * G:(h + 1) * G].double().reshape(G * W, D)
        x = (q @ k.t().contiguous()) / math.sqrt(D)
        if case["causal"]:
            newest = T - W + torch.arange(G * W, device=DEVICE) % W
            x = x.masked_fill(torch.arange(T, device=DEVICE)[None] > newest[:, None], -math.inf)
        p = torch.softmax(x, 1)
        out[l, b, h * G:(h + 1) * G] = (p @ v).reshape(G, W, D)
        lse[l, b, h * G:(h + 1) * G] = torch.logsumexp(x, 1).reshape(G, W)
        if weights is not None:
            weights[unit, :T] = s["weights"][unit, :T].double() + p.sum(0)
    res = {"out": out, "lse": lse}
    return res if weights is None else dict(res, weights_out=weights)


def _exact_rows(s, idx, rows):
    """Rows idx(unit) -> packed; as codes and scales, or as the rows that they stand for."""
    case = s["case"]
    L, N_B, H, D = (case[k] for k in ("layers", "batch", "heads", "dim"))
    lens, out = s["lens"].tolist(), {}
    for name in ("k", "v"):
        value = torch.zeros((L * N_B * H, rows, D), dtype=torch.float64, device=DEVICE)
        scales = torch.zeros((L * N_B * H, _blocks(rows)), dtype=torch.float64, device=DEVICE)
        for unit in range(L * N_B * H):
            l, b, h = unit // (N_B * H), unit // H % N_B, unit % H
            x = _slab(s, name, l, b, h, lens[b])
            x = x if idx is None else x[idx[unit].long()]
            codes, scale = _exact_pack(x[None], case["code"])
            if "back_k" in s:
                codes = codes * scale.repeat_interleave(BLOCK, 1)[:, :codes.shape[1], None]
            value[unit, :x.shape[0]] = codes[0]
            scales[unit, :scale.shape[1]] = scale[0]
        out[name] = value.reshape(L, N_B, H, rows, D)
        if "back_k" not in s:
            out[name + "_scale"] = scales.reshape(L, N_B, H, -1)
    return out


def _exact_recode(s):
    case = s["case"]
    return _exact_rows(s, s["idx"] if case["keep"] else None, case["keep"] or case["length"])


def _exact_evict(s):
    case = s["case"]
    keep, H, L = case["budget"], case["heads"], case["layers"]
    lens = s["lens"].tolist() * L
    chosen, carried = [], torch.zeros_like(s["weights"], dtype=torch.float64)
    for unit in range(_units(case)):
        T = lens[unit // H]
        w = s["weights"][unit, :T].double()
        sinks = min(case["sink"], keep)
        last = min(case["last"], keep - sinks)
        middle = torch.argsort(-w[sinks:T - last], stable=True)[:keep - sinks - last] + sinks
        idx = torch.cat([torch.arange(sinks, device=DEVICE), middle.sort().values, torch.arange(T - last, T, device=DEVICE)])
        carried[unit, :keep] = w[idx]
        chosen.append(idx)
    return dict(_exact_rows(s, chosen, keep), idx=None, n_kept=None, weights=carried)
