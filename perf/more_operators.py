"""A bounded cache in 4 bits and the pages that it lives in, as they are measured: what each operator computes in plain torch, and
the library's calls.

The serving loop between two compression events, with a cache of half the bytes that 8 bits take: new tokens go into it
(`ams_append`), are attended to (`ams_attend`), rows move between it and caches of other element types (`ams_recode`, `ams_evict`),
and the pages of all sequences follow their lengths on the GPU (`ams_assign_pages`).

A cache in 4 bits holds floats of one sign, two exponent and one mantissa bit (magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6), two a byte, the
even channel in the low half, and one byte of scale for every 32 channels of a row: 2^(byte - 127), the least power of two (from 2^-120
on) that takes the largest magnitude of the 32 to 7 or less (7 is as near to 6 as any value of the top binade may be to its code);
0 where all are 0.  The scales of 16 positions lie together, 32 channels after 32 channels: [..., blocks, dim / 32, 16].

A case is a dict:
  kind      "append" | "attend" | "move" | "pages"
  layers, batch, heads, group, dim, dtype ("bf16" | "f32": of queries and of rows that are no codes)
  length, shortest   cache lengths are spread over [shortest, length] (equal: all sequences have that length)
  paged     pages of 16 positions and a block table; else one slab per (layer, sequence, KV head)
  append:   new (tokens per sequence), layout ("half" | "interleaved"), rotated (channels), norm, first (positions begin there)
  attend:   window (queries per head), causal, weights (accumulate them)
  move:     keep (rows that stay), by ("index": a compression event's rows of bf16 or fp32 to 4 bits; "weight": back to the budget, 4 bits
            to 4 bits), sink, last
  pages:    mode ("step": every sequence gets a token; "mixed": some end, some shrink to `keep`, some begin), prompt (tokens
            of those that begin, at most), room (free pages over those asked for)

What a call wrote in 4 bits is read back into rows, within the pass.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
BLOCK = 16
GROUP = 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MOST = 7.0
EPS = 1e-6
BASE = 500000.0


def _case(name, kind, **kw):
    c = dict(kind=kind, layers=1, batch=1, heads=8, group=4, dim=128, dtype="bf16", length=4096, shortest=0, paged=False)
    c.update({"append": dict(new=1, layout="half", rotated=128, norm=True, first=0),
              "attend": dict(window=1, causal=False, weights=True), "move": dict(keep=2048, by="index", sink=4, last=32),
              "pages": dict(mode="step", prompt=0, keep=2048, room=1.2, paged=True)}[kind])
    c.update(kw)
    c["shortest"] = c["shortest"] or c["length"]
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one sequence's next token in one layer
        _case("append-one", "append", length=2177),
        # the next token of 64 sequences in pages; half of the channels rotate, far positions
        _case("append-batch", "append", batch=64, length=4096, shortest=700, paged=True, layout="interleaved", rotated=64, first=200000),
        # a piece of four prompts
        _case("append-prompt", "append", batch=4, length=1111, shortest=640, new=509),
        # one token over one bounded cache: latency
        _case("attend-one", "attend", length=2177),
        # the next token of 64 sequences of 4096 to 16384 positions in pages
        _case("attend-batch", "attend", batch=64, length=16384, shortest=4096, paged=True),
        # one token over a long cache
        _case("attend-long", "attend", heads=4, group=7, length=131072),
        # 32 tokens at once, causal (a draft verified, a window replayed)
        _case("attend-window", "attend", length=32768, window=32, causal=True),
        # fp32 queries, 64 channels, several layers at once
        _case("attend-f32-d64", "attend", layers=6, batch=4, heads=2, group=7, dim=64, dtype="f32", window=2, length=9001, shortest=700,
              causal=True),
        # what a compression event over all layers keeps, into a cache of 4 bits
        _case("move-event", "move", layers=32, length=32768),
        # long caches of a ragged batch in pages back to the budget
        _case("move-evict", "move", by="weight", layers=8, batch=8, heads=4, group=7, length=16384, shortest=6000, paged=True),
        # 64 running sequences, a token each
        _case("pages-step", "pages", batch=64, length=16384, shortest=1000),
        # a large batch between two steps: requests end, caches went back to their budget, prompts begin, and not all find room
        _case("pages-mixed", "pages", batch=768, length=32768, shortest=300, mode="mixed", prompt=4096, room=0.9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attend", "attend", "attend", "move", "pages"))
    if kind == "pages":
        batch, length = _log(rng, 1, 768), _log(rng, 300, 32768)
        mode = rng.choice(("step", "mixed"))
        return _case("", kind, batch=batch, length=length, shortest=max(1, length // rng.choice((1, 3, 20))), mode=mode,
                     prompt=min(length, _log(rng, 16, 4096)) if mode == "mixed" else 0, keep=max(16, length // rng.choice((2, 8))),
                     room=rng.choice((0.5, 0.9, 1.0, 2.0)))
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    heads, group = rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 2, 4, 4, 7, 8))
    dim = rng.choice((64, 128, 128, 128))
    length = _log(rng, 300, 131072) if kind == "attend" else _log(rng, 300, 32768) if kind == "move" else _log(rng, 300, 8192)
    most = (1 << 29) // (length * heads * dim)  # (layer, sequence) pairs: half of the largest listed cache
    if kind == "append":
        most = min(most, 64)
    pairs = max(1, min(_log(rng, 1, 128), most))
    batch = max(1, min(pairs, rng.choice((1, 1, 2, 4, 8, 16, 64))))
    shortest = length if batch == 1 or rng.random() < 0.3 else max(200, int(length * rng.uniform(0.1, 0.9)))
    kw = dict(layers=max(1, pairs // batch) if kind != "append" else 1, batch=batch, heads=heads, group=group, dim=dim, dtype=dtype,
              length=length, shortest=shortest, paged=rng.random() < 0.4)
    if kind == "append":
        new = 1 if rng.random() < 0.5 else min(_log(rng, 2, 512), 4096 // batch, shortest // 2)
        kw.update(new=max(1, new), layout=rng.choice(("half", "interleaved")), norm=rng.random() < 0.7,
                  rotated=rng.choice((dim, dim, dim // 2, 2 * rng.randint(2, dim // 2))), first=rng.choice((0, 0, rng.randint(1, 1000000))))
    elif kind == "attend":
        window = 1 if rng.random() < 0.6 else rng.randint(2, 32)
        if length * batch * kw["layers"] * heads * group * window > 1 << 27:  # the plain form keeps every probability
            window = 1
        kw.update(window=window, causal=rng.random() < 0.7, weights=rng.random() < 0.7)
    else:
        keep = max(32, int(shortest / rng.choice((1.05, 2, 8, 16))))
        kw.update(keep=min(keep, shortest), by=rng.choice(("index", "weight")), sink=rng.choice((0, 4, 16)), last=rng.choice((0, 32, 33)))
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


def _table(lens, seed):
    """Block table over a shuffled pool that holds just these sequences; entries past a sequence's end are -1."""
    counts = [_blocks(n) for n in lens]
    perm = torch.randperm(sum(counts), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lens), max(counts)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = perm[at:at + n]
        at += n
    return table.to(DEVICE), at


def _rows_to_pool(x, table, n_blocks):
    """[B, H, blocks * 16, C] of one layer -> [n_blocks * 16, H, C]."""
    b, j = (table >= 0).nonzero(as_tuple=True)
    pool = torch.zeros((n_blocks, BLOCK, x.shape[1], x.shape[3]), dtype=x.dtype, device=DEVICE)
    pool[table[b, j].long()] = x.unflatten(2, (-1, BLOCK)).transpose(1, 2)[b, j].transpose(1, 2)
    return pool.flatten(0, 1)


def _scales_to_pool(x, table, n_blocks):
    """[B, H, blocks, groups, 16] of one layer -> [n_blocks, H, groups, 16]."""
    b, j = (table >= 0).nonzero(as_tuple=True)
    pool = torch.zeros((n_blocks, x.shape[1]) + x.shape[3:], dtype=x.dtype, device=DEVICE)
    pool[table[b, j].long()] = x.transpose(1, 2)[b, j]
    return pool


def _rows(gen, case, T):
    """Rows of one layer [B, H, T, D], float32: a few loud channels, and tokens of different loudness."""
    shape = (case["batch"], case["heads"], T, case["dim"])
    channel = 1 + 3 * (torch.rand((1, case["heads"], 1, case["dim"]), device=DEVICE, generator=gen) > 0.96)
    token = torch.randn((case["batch"], 1, T, 1), device=DEVICE, generator=gen).mul_(0.3).exp_()
    return torch.randn(shape, device=DEVICE, generator=gen).mul_(channel).mul_(token)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    if case["kind"] == "pages":
        return _prepare_pages(case, seed, gen)
    L, N_B, H, G, D = (case[k] for k in ("layers", "batch", "heads", "group", "dim"))
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    lens, new = _lengths(case), case.get("new", 0)
    s = {"case": case, "lens": torch.tensor(lens, dtype=torch.int32, device=DEVICE), "handle": None}
    table, n_blocks = _table([n + new for n in lens], seed) if case["paged"] else (None, 0)
    s["table"] = table
    T = max(lens) + new
    padded = _blocks(T) * BLOCK
    inside = (torch.arange(padded, device=DEVICE) < s["lens"][:, None])[:, None, :, None]  # [B, 1, rows, 1]
    for name in ("k", "v"):
        rows, scales = [], []
        for _ in range(L):
            x = _rows(gen, case, padded)
            if name == "k" and kind == "attend":  # some stretches are what the recent queries look at
                x[:, :, ::37] *= 1.5
            if kind == "move" and case["by"] == "index":
                x = x.to(dtype)
                rows.append(_rows_to_pool(x, table, n_blocks) if case["paged"] else x)
                continue
            codes, scale = _pack(x.masked_fill_(~inside, 0.0))
            rows.append(_rows_to_pool(codes, table, n_blocks) if case["paged"] else codes)
            scales.append(_scales_to_pool(scale, table, n_blocks) if case["paged"] else scale)
            del x, codes, scale
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
        s["idx"] = (s["lens"][:, None] + torch.arange(new, dtype=torch.int32, device=DEVICE)).repeat_interleave(H, 0).repeat(L, 1)
        s["n_kept"] = torch.full((_units(case),), new, dtype=torch.int32, device=DEVICE)
        s["back_k"] = torch.zeros((L, N_B, H, new, D), dtype=dtype, device=DEVICE)
        s["back_v"] = torch.zeros_like(s["back_k"])
    elif kind == "attend":
        W = case["window"]
        s["q"] = torch.randn((L, N_B, H * G, W, D), device=DEVICE, generator=gen).to(dtype)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((L, N_B, H * G, W), device=DEVICE)
        if case["weights"]:
            s["weights"] = torch.rand((_units(case), T), device=DEVICE, generator=gen).pow_(4) * 3
            s["weights_out"] = torch.zeros_like(s["weights"])
    else:
        keep = case["keep"]
        if case["by"] == "index":
            order = torch.rand((_units(case), T), device=DEVICE, generator=gen)
            order.masked_fill_(~inside[:, 0, :T, 0].repeat_interleave(H, 0).repeat(L, 1), 2.0)
            s["idx"] = order.argsort(1)[:, :keep].sort(1).values.to(torch.int32).contiguous()
            s["n_kept"] = torch.full((_units(case),), keep, dtype=torch.int32, device=DEVICE)
        else:
            s["weights"] = torch.randn((_units(case), T), device=DEVICE, generator=gen).mul_(1.5).exp_()
            s["weights_out"] = torch.zeros_like(s["weights"])
            s["idx"] = torch.full((_units(case), keep), -1, dtype=torch.int32, device=DEVICE)
            s["n_kept"] = torch.zeros(_units(case), dtype=torch.int32, device=DEVICE)
        for name in ("k", "v"):
            s["to_" + name] = torch.zeros((L, N_B, H, keep, D // 2), dtype=torch.uint8, device=DEVICE)
            s["to_" + name + "_scale"] = torch.zeros((L, N_B, H, _blocks(keep), D // GROUP, BLOCK), dtype=torch.uint8, device=DEVICE)
            s["back_" + name] = torch.zeros((L, N_B, H, keep, D), dtype=dtype, device=DEVICE)
    return s


def _prepare_pages(case, seed, gen):
    N_B, T = case["batch"], case["length"]
    had = torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE)
    want, slots = had + 1, N_B
    if case["mode"] == "mixed":  # a tenth end, a tenth begin, a fifth went back to their budget, the others go on
        what = torch.rand(N_B, device=DEVICE, generator=gen)
        prompt = torch.randint(1, case["prompt"] + 1, (N_B,), device=DEVICE, generator=gen, dtype=torch.int32)
        had = torch.where((what >= 0.1) & (what < 0.2), 0, had)
        want = torch.where(what < 0.1, 0, torch.where(what < 0.2, prompt, torch.where(what < 0.4, had.clamp(max=case["keep"]), had + 1)))
        slots = N_B + case["prompt"] * max(1, N_B // 4)  # for as many tokens as a step takes
    s = {"case": case, "handle": None, "had": had, "want": want.to(torch.int32).contiguous()}
    table, used = _table(_lengths(case), seed)
    width = _blocks(T + 1)
    s["table"] = torch.full((N_B, width), -1, dtype=torch.int32, device=DEVICE)
    s["table"][:, :table.shape[1]] = table
    s["table"].masked_fill_(torch.arange(width, device=DEVICE) >= (had[:, None] + BLOCK - 1) // BLOCK, -1)
    asked = ((s["want"] + BLOCK - 1) // BLOCK - (had + BLOCK - 1) // BLOCK).clamp(min=0)
    n_pages = used + 100 + N_B * max(1, _blocks(case["prompt"])) // 2
    free = min(int(int(asked.sum()) * case["room"]), n_pages - used)
    spare = used + torch.randperm(n_pages - used, generator=torch.Generator().manual_seed(seed))[:free].to(torch.int32)
    head = n_pages - free // 2 - 1                     # the ring's free stretch goes round its end
    s["ring"] = torch.full((n_pages,), -1, dtype=torch.int32, device=DEVICE)
    s["ring"][(head + torch.arange(free, device=DEVICE)) % n_pages] = spare.to(DEVICE)
    s["state"] = torch.tensor([head, free], dtype=torch.int32, device=DEVICE)
    s["table_out"], s["state_out"] = torch.zeros_like(s["table"]), torch.zeros_like(s["state"])
    s["lens_out"] = torch.zeros_like(had)
    s["starts"] = torch.zeros(N_B + 1, dtype=torch.int32, device=DEVICE)
    s["slots"] = torch.zeros(slots, dtype=torch.int64, device=DEVICE)
    return s


# ---------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _own(s)
    return {"append": _append, "attend": _attend, "move": _move, "pages": _pages}[s["case"]["kind"]](s)


def _own(s):
    from paper_2605_23200_amd import binding as B
    case, kind = s["case"], s["case"]["kind"]
    if s["handle"] is None:
        s["handle"] = _handle(B, s)
    h = s["handle"]
    if kind == "append":
        B.ams_append(h["p"], s["new_q"], s["new_k"], s["new_v"], s["q_weight"], s["k_weight"], EPS, h["rope"], s["first"],
                     s["lens"], s["q_out"], h["cache"], s["lens_out"])
        B.ams_recode(h["p_back"], h["cache"], None, h["back"], s["idx"], s["n_kept"])
        return {"q": s["q_out"], "lens": s["lens_out"], "k": s["back_k"], "v": s["back_v"]}
    if kind == "attend":
        B.ams_attend(h["p"], h["cache"], s["lens"], s["q"], s["out"], h["ws"], s["lse"], s.get("weights"), s.get("weights_out"))
        return {k: s[k] for k in ("out", "lse", "weights_out") if k in s}
    if kind == "pages":
        B.ams_assign_pages(h["p"], s["had"], s["want"], s["table"], s["table_out"], s["ring"], s["state"], s["state_out"],
                           s["starts"], s["slots"], s["lens_out"])
        return {k: s[k] for k in ("table_out", "ring", "state_out", "starts", "slots", "lens_out")}
    if case["by"] == "index":
        B.ams_recode(h["p"], h["cache"], None, h["to"], s["idx"], s["n_kept"])
        B.ams_recode(h["p_back"], h["to"], h["kept"], h["back"])
        return {"k": s["back_k"], "v": s["back_v"]}
    B.ams_evict(h["p"], h["cache"], s["lens"], s["weights"], h["to"], s["weights_out"], s["idx"], s["n_kept"], h["ws"], h["kept"])
    B.ams_recode(h["p_back"], h["to"], h["kept"], h["back"])
    return {"k": s["back_k"], "v": s["back_v"], "idx": s["idx"], "n_kept": s["n_kept"], "weights": s["weights_out"]}


def _handle(B, s):
    """What a user's program keeps from call to call: parameters, views, the rotation's table, the workspace."""
    case, kind = s["case"], s["case"]["kind"]
    common = dict(n_layers=case["layers"], batch=case["batch"], n_kv_heads=case["heads"], group=case["group"],
                  window=case.get("window", 1), head_dim=case["dim"], kv_dtype=B.F32 if case["dtype"] == "f32" else B.BF16, n_segments=1)
    if kind == "pages":
        return {"p": B.make_params(t_max=case["length"] + 1, budget=1, **common)}
    T = case["length"] + case.get("new", 0)
    kept = case.get("keep", T)
    h = {"p": B.make_params(t_max=T, budget=kept, causal=case.get("causal", False), n_sink=case.get("sink", 0),
                            n_last=case.get("last", 0), **common)}
    h["cache"] = B.cache_view(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"), block_table=s["table"])
    if kind == "append":
        h["rope"] = B.make_rope(case["rotated"], layout=B.ROPE_HALF if case["layout"] == "half" else B.ROPE_INTERLEAVED, base=BASE)
        h["back"] = B.cache_view(s["back_k"], s["back_v"])
        h["p_back"] = B.make_params(t_max=T, budget=case["new"], **common)
    if kind == "attend":
        h["ws"] = torch.empty(B.ams_attend_workspace_bytes(h["p"]), dtype=torch.uint8, device=DEVICE)
    if kind == "move":
        if case["by"] == "weight":
            h["ws"] = torch.empty(B.ams_evict_workspace_bytes(h["p"]), dtype=torch.uint8, device=DEVICE)
        h["kept"] = torch.full((case["batch"],), kept, dtype=torch.int32, device=DEVICE)
        h["to"] = B.cache_view(s["to_k"], s["to_v"], s["to_k_scale"], s["to_v_scale"])
        h["back"] = B.cache_view(s["back_k"], s["back_v"])
        h["p_back"] = B.make_params(t_max=kept, budget=kept, **common)
    return h


# ---- the plain forms ----

def _pack(x):
    """Rows [..., T, D] in 32 or 64 bits -> bytes [..., T, D / 2] and scales [..., blocks, D / 32, 16]."""
    T, D = x.shape[-2:]
    y = x.unflatten(-1, (-1, GROUP))
    byte = _scale_byte(y.abs().amax(-1))                                     # [..., T, D / 32]
    y = y * _power(-byte, x.dtype)[..., None]
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for edge, tie in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):  # ties to the even code
        code += (a >= edge) if tie else (a > edge)
    code += 8 * (y < 0)
    code = code.flatten(-2)
    scale = torch.nn.functional.pad(byte.to(torch.uint8), (0, 0, 0, -T % BLOCK)).unflatten(-2, (-1, BLOCK)).transpose(-1, -2)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.contiguous()


def _scale_byte(largest):
    m, e = torch.frexp(largest)
    power = (e - 3 + (m > MOST / 8)).clamp(min=-120)
    return torch.where(largest > 0, power + 127, 0)


def _power(byte, dtype):
    """2^(byte - 127), and 2^(127 + byte) for negated ones; 0 stands for 0 either way."""
    e = torch.where(byte < 0, byte + 127, byte - 127)
    return torch.where(byte == 0, 0.0, torch.ldexp(torch.ones((), dtype=dtype, device=DEVICE), e))


def _unpack(codes, scale):
    """Bytes [..., T, D / 2], scales [..., blocks, D / 32, 16] -> rows [..., T, D] in float32."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEVICE)
    pair = torch.stack([level.repeat(16), level.repeat_interleave(16)], 1)   # by the byte: low half, high half
    x = pair[codes.int()].flatten(-2)
    power = _power(scale.int(), torch.float32).transpose(-1, -2).flatten(-3, -2)[..., :x.shape[-2], :]
    return x.unflatten(-1, (-1, GROUP)).mul_(power[..., None]).flatten(-2)


def _values(s, name):
    """A cache's rows [L, B, H, T, D] in float32."""
    if s["table"] is None:
        return _unpack(s[name], s[name + "_scale"])
    page = s["table"].long().clamp(min=0)
    codes = s[name].unflatten(1, (-1, BLOCK))[:, page].movedim(4, 2).flatten(3, 4)   # [L, B, blocks, 16, H, C] -> [L, B, H, T, C]
    return _unpack(codes, s[name + "_scale"][:, page].movedim(3, 2))


def _picked(s, name, idx):
    """Rows idx [units, n] of a cache, [L, B, H, n, D], in float32."""
    case = s["case"]
    L, N_B, H = case["layers"], case["batch"], case["heads"]
    t = idx.long().reshape(L, N_B, H, -1)
    l, b, h = (torch.arange(n, device=DEVICE).reshape(shape) for n, shape in
               ((L, (-1, 1, 1, 1)), (N_B, (1, -1, 1, 1)), (H, (1, 1, -1, 1))))
    if s["table"] is None:
        x, block = s[name][l, b, h, t], (l, b, h, t // BLOCK)
    else:
        page = s["table"].long()[b, t // BLOCK]
        x, block = s[name][l, page * BLOCK + t % BLOCK, h], (l, page, h)
    if name + "_scale" not in s:
        return x.float()
    byte = s[name + "_scale"][block].gather(-1, (t % BLOCK)[..., None, None].expand(*t.shape, case["dim"] // GROUP, 1))  # [..., D / 32, 1]
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEVICE)
    x = torch.stack([level[(x & 15).int()], level[(x >> 4).int()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, GROUP)) * _power(byte.int(), torch.float32)).flatten(-2)


def _normed(x, weight):
    if weight is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)


def _turned(x, cos, sin, case):
    """x [L, B, W, heads, D]; cos, sin [B, W, 1, rotated / 2]."""
    n = case["rotated"]
    cos, sin = cos.to(x.dtype), sin.to(x.dtype)
    if case["layout"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., n:]], -1)


def _append(s):
    case, new, n = s["case"], s["case"]["new"], s["case"]["rotated"]
    pos = s["first"].double()[:, None] + torch.arange(new, device=DEVICE)
    angle = pos[..., None, None] * BASE ** (-torch.arange(0, n, 2, dtype=torch.float64, device=DEVICE) / n)
    cos, sin = angle.cos(), angle.sin()
    q = _turned(_normed(s["new_q"].float(), s["q_weight"]), cos, sin, case).to(s["q_out"].dtype).movedim(3, 2).contiguous()
    # keys in 64 bits: a code moves by a step where the value crosses the middle between two
    rows = {"k": _turned(_normed(s["new_k"].double(), s["k_weight"]), cos, sin, case), "v": s["new_v"].float()}
    at = s["lens"].long()[:, None] + torch.arange(new, device=DEVICE)        # [B, W] rows written
    b = torch.arange(case["batch"], device=DEVICE)[:, None]
    out = {"q": q, "lens": s["lens"] + new}
    for name, x in rows.items():
        codes, scale = _pack(x.movedim(3, 2).unsqueeze(-2))                  # [L, B, H, W, 1, D / 2], [L, B, H, W, 1, D / 32, 16]
        codes, scale = codes[..., 0, :], scale[..., 0, :, 0]
        if s["table"] is None:
            s[name][:, b, :, at] = codes.movedim((1, 3), (0, 1))
            s[name + "_scale"][:, b, :, at // BLOCK, :, at % BLOCK] = scale.movedim((1, 3), (0, 1))
        else:
            page = s["table"].long()[b, at // BLOCK]
            s[name][:, page * BLOCK + at % BLOCK] = codes.movedim(2, 3)
            s[name + "_scale"][:, page, :, :, at % BLOCK] = scale.movedim((1, 3), (0, 1))
        out[name] = _picked(s, name, s["idx"]).to(s["q_out"].dtype)
    return out


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


def _move(s):
    case = s["case"]
    if case["by"] == "index":
        return {name: _unpack(*_pack(_picked(s, name, s["idx"]))).to(s["back_k"].dtype) for name in ("k", "v")}
    w, keep, H, L = s["weights"], case["keep"], case["heads"], case["layers"]
    lens = s["lens"].repeat_interleave(H).repeat(L)[:, None]
    t = torch.arange(w.shape[1], device=DEVICE)
    sinks = min(case["sink"], keep)
    always = (t < sinks) | (t >= lens - min(case["last"], keep - sinks))
    rank = torch.where(t < lens, torch.where(always, math.inf, w), -math.inf)
    idx = rank.sort(dim=1, descending=True, stable=True).indices[:, :keep].sort(1).values
    out = {name: _picked(s, name, idx).to(s["back_k"].dtype) for name in ("k", "v")}
    carried = torch.zeros_like(w)
    carried[:, :keep] = w.gather(1, idx)
    n_kept = torch.full((w.shape[0],), keep, dtype=torch.int32, device=DEVICE)
    return dict(out, idx=idx.to(torch.int32), n_kept=n_kept, weights=carried)


def _pages(s):
    had, want, n_pages = s["had"].long(), s["want"].long(), s["ring"].numel()
    head, count = s["state"].long()
    pages_had, pages_want = (had + BLOCK - 1) // BLOCK, (want + BLOCK - 1) // BLOCK
    asked = (pages_want - pages_had).clamp(min=0)
    first = asked.cumsum(0) - asked
    served = (asked == 0) | (first + asked <= count)                         # in order, as far as the free pages go
    freed = (pages_had - pages_want).clamp(min=0)
    first_freed = freed.cumsum(0) - freed
    j = torch.arange(s["table"].shape[1], device=DEVICE)[None]
    taken = served[:, None] & (j >= pages_had[:, None]) & (j < pages_want[:, None])
    stay = j < torch.where(served, torch.minimum(pages_had, pages_want), pages_had)[:, None]
    fresh = s["ring"][(head + first[:, None] + j - pages_had[:, None]) % n_pages]
    table = torch.where(taken, fresh, torch.where(stay, s["table"], -1))
    gone = (j >= pages_want[:, None]) & (j < pages_had[:, None])
    place = torch.where(gone, (head + count + first_freed[:, None] + j - pages_want[:, None]) % n_pages, n_pages)
    ring = torch.cat([s["ring"], s["ring"][:1]])                             # (one place more, for the entries that stay)
    ring[place] = s["table"]
    ring = ring[:-1]
    used = (asked * served).sum()
    state = torch.stack([(head + used) % n_pages, count - used + freed.sum()])
    new = (want - had).clamp(min=0)
    starts = torch.cat([new.new_zeros(1), new.cumsum(0)])
    i = torch.arange(s["slots"].numel(), device=DEVICE)
    owner = torch.searchsorted(starts, i, right=True).sub_(1).clamp_(max=had.numel() - 1)
    pos = had[owner] + i - starts[owner]
    page = table[owner, (pos // BLOCK).clamp(max=table.shape[1] - 1)].long()
    slots = torch.where((i < starts[-1]) & served[owner], page * BLOCK + pos % BLOCK, -1)
    return {"table_out": table, "ring": ring, "state_out": state.to(torch.int32), "starts": starts.to(torch.int32), "slots": slots,
            "lens_out": torch.where(served, want, had).to(torch.int32)}


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    L, N_B, H, G, D = (case[k] for k in ("layers", "batch", "heads", "group", "dim"))
    lens = _lengths(case)
    row = D / 2 + D / GROUP                                      # of a row in 4 bits, with its scales
    if case["kind"] == "pages":
        table = 4 * N_B * _blocks(case["length"] + 1)
        slots = N_B if case["mode"] == "step" else N_B + case["prompt"] * max(1, N_B // 4)
        return {"bytes": 2 * table + 8 * slots + 16 * N_B, "flops": table + slots}
    if case["kind"] == "append":
        new = L * N_B * case["new"]
        read = new * (G + 2) * H * D * e
        return {"bytes": read + new * (G * H * D * e + 2 * H * (2 * row + D * e)), "flops": new * (G + 1) * H * D * 8}
    if case["kind"] == "attend":
        n, tokens = G * case["window"], L * H * sum(lens)
        rows = L * N_B * H * n
        return {"bytes": tokens * (2 * row + (8 if case["weights"] else 0)) + rows * (2 * D * e + 4), "flops": 4 * tokens * n * D}
    kept = _units(case) * case["keep"]
    if case["by"] == "index":
        return {"bytes": kept * (2 * (2 * D * e + 2 * row) + 4), "flops": kept * 2 * D * 4}
    return {"bytes": L * H * sum(lens) * 4 + kept * (2 * (3 * row + D * e) + 12), "flops": L * H * sum(lens) + kept * 2 * D}


# ---------------------------------------------------------------------------------------------------------------
# The same outputs in 64 bits, unit by unit
# ---------------------------------------------------------------------------------------------------------------

def _exact_rounded(x):
    """Rows [n, D] in float64 -> the values that their 4 bits stand for."""
    y = x.reshape(x.shape[0], -1, GROUP)
    largest = y.abs().amax(-1, keepdim=True)
    power = torch.floor(torch.log2(largest.clamp(min=1e-300) / MOST)) - 1
    for _ in range(3):
        power = torch.where(largest > MOST * torch.exp2(power), power + 1, power)
    scale = torch.exp2(power.clamp(min=-120))
    y = y / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)   # 1/2 below 2, then 1, then 2
    y = (torch.round(y / step) * step).clamp(-6, 6) * scale
    return torch.where(largest > 0, y, 0.0).reshape(x.shape)


def _slab(s, name, l, b, h, T):
    """Rows 0 .. T of one unit, float64."""
    D, n = s["case"]["dim"], _blocks(T)
    if s["table"] is None:
        x, scale = s[name][l, b, h, :T], s[name + "_scale"][l, b, h, :n] if name + "_scale" in s else None
    else:
        page = s["table"][b, :n].long()
        x = s[name][l].reshape(-1, BLOCK, s["case"]["heads"], s[name].shape[-1])[page, :, h].flatten(0, 1)[:T]
        scale = s[name + "_scale"][l, page, h] if name + "_scale" in s else None
    if scale is None:
        return x.double()
    value = torch.zeros((T, D), dtype=torch.float64, device=DEVICE)
    for half in (0, 1):
        code = (x.int() >> (4 * half)) & 15
        e, m = (code >> 1) & 3, (code & 1).double()
        size = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e.double() - 1))
        value[:, half::2] = torch.where(code > 7, -size, size)
    power = torch.exp2(scale.double() - 127) * (scale > 0)                   # [n, D / 32, 16]
    return value * power.transpose(1, 2).reshape(n * BLOCK, -1)[:T].repeat_interleave(GROUP, 1)


def exact(case, seed):
    if case["kind"] == "pages":
        return None
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "move": _exact_move}[case["kind"]](s)


def _exact_append(s):
    case = s["case"]
    N_B, D, new, n = (case[k] for k in ("batch", "dim", "new", "rotated"))
    first, second = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
    f = torch.tensor([BASE ** (-2 * i / n) for i in range(n // 2)], dtype=torch.float64, device=DEVICE)
    q = torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEVICE)
    out = {name: torch.zeros(s["back_k"].shape, dtype=torch.float64, device=DEVICE) for name in ("k", "v")}
    for b in range(N_B):
        z = torch.polar(torch.ones((new, n // 2), dtype=torch.float64, device=DEVICE),
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
            out[name][0, b] = _exact_rounded(rows[name].reshape(-1, D)).reshape(rows[name].shape).transpose(0, 1)
    return dict(out, q=q, lens=None)


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


def _exact_move(s):
    case = s["case"]
    keep, H, N_B, D = case["keep"], case["heads"], case["batch"], case["dim"]
    lens = s["lens"].tolist()
    out = {name: torch.zeros((_units(case), keep, D), dtype=torch.float64, device=DEVICE) for name in ("k", "v")}
    carried = torch.zeros_like(s["weights"], dtype=torch.float64) if case["by"] == "weight" else None
    for unit in range(_units(case)):
        l, b, h = unit // (N_B * H), unit // H % N_B, unit % H
        T = lens[b]
        if case["by"] == "index":
            idx = s["idx"][unit].long()
        else:
            w = s["weights"][unit, :T].double()
            sinks = min(case["sink"], keep)
            last = min(case["last"], keep - sinks)
            middle = torch.argsort(-w[sinks:T - last], stable=True)[:keep - sinks - last] + sinks
            idx = torch.cat([torch.arange(sinks, device=DEVICE), middle.sort().values, torch.arange(T - last, T, device=DEVICE)])
            carried[unit, :keep] = w[idx]
        for name in ("k", "v"):
            x = _slab(s, name, l, b, h, T)[idx]
            out[name][unit] = _exact_rounded(x) if case["by"] == "index" else x
    out = {name: x.reshape(s["back_k"].shape) for name, x in out.items()}
    return out if carried is None else dict(out, idx=None, n_kept=None, weights=carried)
