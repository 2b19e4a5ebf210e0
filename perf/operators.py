"""What is measured of the operators for serving in 8 bits: the K/V cache with a scale for each block of tokens and head, the tables
and slot maps that an engine keeps on the GPU, and the projections over 8-bit integers.

`listed()` names twelve cases and `draw()` picks more from the same ranges; `prepare()` makes what a serving program holds before the
call, `run()` is one pass: in plain torch operations, or, where `own` is true, through `paper_2509_16495_amd.binding`.  A case is a
dict of plain values; its `kind` says which path it takes:

  tables   request lengths -> block tables, slot map and row offsets of a step, then the same tokens given back
  append   new K/V rows into the scaled FP8 cache
  decode   one new token per sequence over that cache, with its append
  prefill  prompts, or chunks behind cached tokens, over that cache, with their append
  mixed    chunks and decode rows in one call, with their append
  proj     activations quantised to int8 token by token, the q|k|v projection into the send buffers, the output projection

Head geometries are those of the models the repository serves (64q/8kv, 40q/8kv, 32q/8kv, 32q/4kv, head_dim 128) split over P
GPUs.  Lengths come from the case's own `lens_seed`, so every preparation of a case has the same amount of work; values and block
tables come from the preparation's seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16
DEVICE = "cuda:0"
FP8 = torch.float8_e4m3fn
E_MIN, E_MAX = -100, 119   # exponents of a block's scale

# (query heads, KV heads, d_model) of the served models
MODELS = ((64, 8, 8192), (64, 8, 5120), (40, 8, 5120), (32, 8, 4096), (32, 4, 2048))
GPU_HEADS = ((8, 1), (8, 1), (4, 1), (5, 1), (16, 2), (10, 2))   # (query, KV) heads on one GPU


def listed():
    return [
        # a decode step's tables: one token more for each of 61 requests, the smallest call there is
        dict(name="tables_decode_61", kind="tables", chunks=0, len_lo=0, len_hi=0, cached=0, decs=61, ctx_lo=1, ctx_hi=8192, P=1, lens_seed=1),
        # admission of a burst of prompts next to a running batch, rows padded for eight ranks
        dict(name="tables_prompts_29", kind="tables", chunks=29, len_lo=1, len_hi=9000, cached=0, decs=256, ctx_lo=1, ctx_hi=8192, P=8, lens_seed=2),
        # the rows of a decode step, each into a block that other tokens share
        dict(name="append_97_tokens", kind="append", chunks=0, len_lo=0, len_hi=0, cached=0, decs=97, ctx_lo=1, ctx_hi=16000, hq=8, hkv=1, D=128,
             dtype="bf16", lens_seed=3),
        # prompts of a large prefill, ragged
        dict(name="append_prompts", kind="append", chunks=23, len_lo=1, len_hi=6000, cached=0, decs=0, ctx_lo=0, ctx_hi=0, hq=16, hkv=2, D=128,
             dtype="bf16", lens_seed=4),
        # interactive decoding: a handful of sequences, latency counts
        dict(name="decode_4_seqs", kind="decode", chunks=0, len_lo=0, len_hi=0, cached=0, decs=4, ctx_lo=1900, ctx_hi=6300, hq=8, hkv=1, D=128,
             dtype="bf16", lens_seed=5),
        # throughput decoding of a 70B shard
        dict(name="decode_256_seqs", kind="decode", chunks=0, len_lo=0, len_hi=0, cached=0, decs=256, ctx_lo=512, ctx_hi=8192, hq=8, hkv=1, D=128,
             dtype="bf16", lens_seed=6),
        # fp32 activations and 64-wide heads: a small model checked at full precision
        dict(name="decode_fp32_heads_of_64", kind="decode", chunks=0, len_lo=0, len_hi=0, cached=0, decs=16, ctx_lo=100, ctx_hi=1500, hq=4, hkv=1, D=64,
             dtype="f32", lens_seed=7),
        # chunks of two long prompts
        dict(name="prefill_2_chunks", kind="prefill", chunks=2, len_lo=900, len_hi=1100, cached=16000, decs=0, ctx_lo=0, ctx_hi=0, hq=8, hkv=1, D=128,
             dtype="bf16", lens_seed=8),
        # conversation serving: one chunk continues a prompt while other sequences decode
        dict(name="mixed_step", kind="mixed", chunks=1, len_lo=1000, len_hi=1000, cached=20000, decs=97, ctx_lo=1000, ctx_hi=16000, hq=8, hkv=1, D=128,
             dtype="bf16", lens_seed=9),
        # projections of a decode step
        dict(name="proj_19_rows", kind="proj", T=19, pad=0, P=8, h=64, h_kv=8, d_model=8192),
        # projections of a chunked-prefill step, ragged
        dict(name="proj_701_rows", kind="proj", T=701, pad=1, P=8, h=64, h_kv=8, d_model=5120),
        # projections of a large prefill
        dict(name="proj_8192_rows", kind="proj", T=8192, pad=0, P=8, h=64, h_kv=8, d_model=8192),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tables", "append", "decode", "decode", "prefill", "mixed", "proj", "proj"])
    seed = rng.randrange(1 << 30)
    none = dict(chunks=0, len_lo=0, len_hi=0, cached=0, decs=0, ctx_lo=0, ctx_hi=0, lens_seed=seed)
    if kind == "proj":
        h, h_kv, d_model = rng.choice(MODELS)
        if rng.random() < 0.25 and h != 40:  # the shift configuration: this GPU's head shard of the weights, nothing to exchange
            h, h_kv, P = h // 8, 1, 1
        else:
            P = rng.choice([4, 8, 8])
        return dict(kind=kind, T=_log_int(rng, 1, 6000), pad=0 if P == 1 else rng.choice([0, 1]), P=P, h=h, h_kv=h_kv, d_model=d_model)
    chunks, hi = _log_int(rng, 1, 40), _log_int(rng, 20, 9000)
    decs, ctx = _log_int(rng, 1, 300), _log_int(rng, 40, 16000)
    if kind == "tables":
        return dict(none, kind=kind, P=rng.choice([1, 2, 8]), chunks=rng.choice([0, chunks]), len_lo=1, len_hi=hi, cached=rng.choice([0, 37, 1024]),
                    decs=decs, ctx_lo=1, ctx_hi=ctx)
    heads = rng.choice(GPU_HEADS)
    shape = dict(none, kind=kind, hq=heads[0], hkv=heads[1], D=128, dtype="bf16")
    if rng.random() < 0.15:
        shape.update(hq=4, hkv=1, D=64, dtype=rng.choice(["bf16", "f32"]))
    small = shape["D"] == 64
    decs = min(decs, 20) if small else decs
    ctx = min(ctx, 1500 if small else 1_100_000 // (decs * shape["hkv"]))
    if kind == "append":
        chunks = min(chunks, max(1, 60000 // hi))
        return dict(shape, chunks=rng.choice([0, chunks]), len_lo=max(1, hi // 8), len_hi=hi, cached=rng.choice([0, 0, 75]), decs=decs, ctx_lo=1, ctx_hi=ctx)
    if kind == "decode":
        return dict(shape, decs=decs, ctx_lo=max(1, ctx // rng.choice([2, 4, 16])), ctx_hi=ctx)
    hi = min(hi, 300 if small else 4000)
    cached = rng.choice([0, 0, _log_int(rng, 100, 500 if small else 16000)])
    chunks = min(chunks, 3 if small or cached else max(1, 12000 // hi))
    if cached:
        hi = min(hi, 1100)
    shape.update(chunks=chunks, len_lo=max(1, hi // rng.choice([1, 2, 8])), len_hi=hi, cached=cached)
    if kind == "mixed":
        shape.update(decs=decs, ctx_lo=max(1, ctx // 8), ctx_hi=ctx)
    return shape


# ---- sizes of a case ---------------------------------------------------------------------------------------------------
def _lengths(case):
    """(new tokens, tokens with them) per sequence: chunks and prompts first, then decode rows."""
    r = random.Random(case["lens_seed"])
    lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["chunks"])]
    return ([(n, n + case["cached"]) for n in lens] + [(1, r.randint(case["ctx_lo"], case["ctx_hi"])) for _ in range(case["decs"])])


def _up(n, m):
    return (n + m - 1) // m * m


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _kv_heads_here(P, h_kv):
    return h_kv // P if h_kv >= P else 1


def work(case):
    kind = case["kind"]
    if kind == "proj":
        T, d, N, K = case["T"], case["d_model"], (case["h"] + 2 * case["h_kv"]) * 128, case["h"] * 128
        send = case["P"] * (T + case["pad"]) * (case["h"] // case["P"] + 2 * _kv_heads_here(case["P"], case["h_kv"])) * 128
        return {"bytes": (N * d + d * K) + 4 * (N + d) + 3 * T * (d + K) + 8 * T + 2 * send + 2 * T * d, "flops": 2 * T * d * (N + K)}
    lens = _lengths(case)
    rows = sum(n for n, _ in lens)
    if kind == "tables":
        new_blocks = sum(_blocks(c) - _blocks(c - n) for n, c in lens)
        return {"bytes": 8 * _up(rows, case["P"]) + 16 * new_blocks + 28 * len(lens), "flops": 0}
    hq, hkv, D, e = case["hq"], case["hkv"], case["D"], 2 if case["dtype"] == "bf16" else 4
    by = rows * (2 * hkv * D * (e + 1) + 8) + sum(_blocks(c) - (c - n) // BLOCK for n, c in lens) * hkv * 8
    if kind == "append":
        return {"bytes": by, "flops": 0}
    cached = sum((c - n) * 2 * hkv * D + _blocks(c - n) * hkv * 8 for n, c in lens)
    return {"bytes": by + cached + rows * 2 * hq * D * e, "flops": 4 * D * hq * sum(n * (c - n) + n * (n + 1) // 2 for n, c in lens)}


# ---- preparation -------------------------------------------------------------------------------------------------------
def _normal(shape, dtype, gen, std=1.0):
    return torch.empty(shape, dtype=dtype, device=DEVICE).normal_(0.0, std, generator=gen)


def _rows(shape, dtype, gen):
    """Activations of a layer: tokens of different magnitude, so that blocks of tokens want different scales."""
    x = _normal(shape, torch.float32, gen)
    return x.mul_(_normal((shape[0],) + (1,) * (len(shape) - 1), torch.float32, gen, 0.7).exp_()).to(dtype)


def _layout(case, gen):
    """Lengths and block tables on the GPU, and how many blocks there are."""
    lens = _lengths(case)
    total = torch.tensor([c for _, c in lens], dtype=torch.int64, device=DEVICE)
    need = (total + BLOCK - 1) // BLOCK
    wide, used = int(need.max()), int(need.sum())
    num_blocks = used + used // 8 + 1
    order = torch.randperm(num_blocks, generator=gen, device=DEVICE).to(torch.int32)
    i = torch.arange(wide, device=DEVICE)
    at = (need.cumsum(0) - need)[:, None] + i
    table = torch.where(i < need[:, None], order[at.clamp(max=num_blocks - 1)], -1)
    return lens, total, table, num_blocks, order, used


def _slots(lens, total, table):
    """Slot of every new token, sequence by sequence."""
    n = torch.tensor([n for n, _ in lens], device=DEVICE)
    s = torch.repeat_interleave(torch.arange(len(lens), device=DEVICE), n)
    p = torch.arange(s.numel(), device=DEVICE) - (n.cumsum(0) - n)[s] + (total - n)[s]
    return table[s, p // BLOCK].long() * BLOCK + p % BLOCK


def _power(e):
    """2^e in float32, -126 <= e <= 127 (from its bits: a power function may be off by a rounding)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale_of(top):
    """Scale of a block whose largest finite magnitude is `top`: the least power of two that brings it to at most 448."""
    e = torch.log2(top.clamp(min=2.0 ** -100) / 448).floor().to(torch.int32)
    e = torch.where(448.0 * _power(e) < top, e + 1, e)
    e = torch.where(448.0 * _power(e - 1) >= top, e - 1, e)
    return _power(e.clamp(E_MIN, E_MAX))


def _codes(x):
    return x.clamp(-448.0, 448.0).to(FP8).view(torch.uint8)


def _prepare_cache(case, seed, gen):
    lens, total, table, num_blocks, _, _ = _layout(case, gen)
    hkv, D = case["hkv"], case["D"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    st = {"kind": case["kind"], "scale": 1.0 / math.sqrt(D), "table": table, "slots": _slots(lens, total, table), "seq_lens": total.to(torch.int32)}
    # what earlier steps left: the tokens in front of the new ones
    cached = torch.tensor([c - n for n, c in lens], device=DEVICE)
    filled = torch.zeros(num_blocks, dtype=torch.int64, device=DEVICE)
    i = torch.arange(table.shape[1], device=DEVICE) * BLOCK
    here = table >= 0
    filled[table[here].long()] = (cached[:, None] - i).clamp(0, BLOCK)[here]
    st["cache"] = torch.zeros((num_blocks, hkv, 2, BLOCK * D), dtype=torch.uint8, device=DEVICE)
    st["scales"] = torch.zeros((num_blocks, hkv, 2), dtype=torch.float32, device=DEVICE)
    step = 1 << 14
    for b in range(0, num_blocks, step):
        n = min(step, num_blocks - b)
        there = (torch.arange(BLOCK, device=DEVICE) < filled[b:b + n, None])[:, None, None, :, None]
        x = _normal((n, hkv, 2, BLOCK, D), torch.float32, gen) * _normal((n, 1, 1, BLOCK, 1), torch.float32, gen, 0.7).exp_() * there
        s = _scale_of(x.abs().amax((3, 4)))
        x = _codes(x / s[..., None, None])
        st["cache"][b:b + n, :, 0] = x[:, :, 0].reshape(n, hkv, BLOCK * D)
        st["cache"][b:b + n, :, 1] = x[:, :, 1].transpose(2, 3).reshape(n, hkv, BLOCK * D)
        st["scales"][b:b + n] = s
    rows = _rows((sum(n for n, _ in lens), case["hq"] + 2 * hkv, D), dtype, gen)   # the fused rows that the exchange delivers
    st["k"], st["v"] = rows[:, case["hq"]:case["hq"] + hkv], rows[:, case["hq"] + hkv:]
    if case["kind"] == "append":
        return st
    st["q"] = rows[:, :case["hq"]]
    st["out"] = torch.empty((rows.shape[0], case["hq"], D), dtype=dtype, device=DEVICE)
    pre, dec = lens[:case["chunks"]], lens[case["chunks"]:]
    st["n_pre"], st["max_q"] = len(pre), max([n for n, _ in pre], default=0)
    st["max_pre"], st["max_dec"] = max([c for _, c in pre], default=0), max([c for _, c in dec], default=0)
    st["q_rows"] = sum(n for n, _ in pre)
    cu = [0]
    for n, _ in pre:
        cu.append(cu[-1] + n)
    st["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEVICE)
    st["num_dec"], st["ws"] = len(dec), None
    return st


def _prepare_tables(case, seed, gen):
    lens, total, table, num_blocks, order, used = _layout(case, gen)
    new = torch.tensor([n for n, _ in lens], dtype=torch.int32, device=DEVICE)
    had = total.to(torch.int32) - new
    i = torch.arange(table.shape[1], device=DEVICE)
    kept = i < ((had + BLOCK - 1) // BLOCK)[:, None]
    table = torch.where(kept, table, -1)
    taken_ids = torch.zeros(num_blocks, dtype=torch.bool, device=DEVICE)
    taken_ids[table[kept].long()] = True
    free = order[~taken_ids[order.long()]].flip(0)
    rows = sum(n for n, _ in lens)
    st = {"kind": "tables", "new": new, "lens": had.contiguous(), "before": had.clone(), "table": table.contiguous(), "n_pre": case["chunks"],
          "q_rows": sum(n for n, _ in lens[:case["chunks"]]), "cu": torch.zeros(case["chunks"] + 1, dtype=torch.int32, device=DEVICE),
          "slots": torch.empty(_up(rows, case["P"]), dtype=torch.int64, device=DEVICE), "taken": torch.empty_like(new), "ws": None}
    st["free"] = torch.cat([free, torch.zeros(num_blocks - free.numel(), dtype=torch.int32, device=DEVICE)])
    st["count"] = torch.tensor([free.numel()], dtype=torch.int32, device=DEVICE)
    return st


def _quantise_rows(x):
    """Rows -> int8 codes and a scale per row."""
    top = x.abs().amax(-1, keepdim=True).float()
    tiny = top < 2.0 ** -100
    inv = torch.where(tiny, 1.0, 127.0 / top)
    # the product of a bf16 value and a float32 one is exact in 64 bits: nearest code, ties to the even one
    return (x.double() * inv.double()).round_().to(torch.int8), torch.where(tiny, 1.0, top / 127.0).squeeze(-1)


def _prepare_proj(case, seed, gen):
    P, h, h_kv, d, T = case["P"], case["h"], case["h_kv"], case["d_model"], case["T"]
    Tp, N, K = T + case["pad"], (h + 2 * h_kv) * 128, h * 128
    st = {"kind": "proj", "P": P, "h": h, "h_kv": h_kv, "x": _rows((T, d), torch.bfloat16, gen), "recv": _rows((P, Tp, h // P, 128), torch.bfloat16, gen),
          "ws": None}
    for name, shape in (("qkv", (N, d)), ("o", (d, K))):   # a checkpoint's weights are quantised once, when they are loaded
        st["w_" + name], st["ws_" + name] = _quantise_rows(_normal(shape, torch.bfloat16, gen, 0.02))
    st["xc"], st["xs"] = torch.empty((T, d), dtype=torch.int8, device=DEVICE), torch.empty(T, dtype=torch.float32, device=DEVICE)
    st["rc"], st["rs"] = torch.zeros(st["recv"].shape, dtype=torch.int8, device=DEVICE), torch.empty(T, dtype=torch.float32, device=DEVICE)
    st["send"] = torch.empty((P, Tp, h // P + 2 * _kv_heads_here(P, h_kv), 128), dtype=torch.bfloat16, device=DEVICE)
    st["out"] = torch.empty((T, d), dtype=torch.bfloat16, device=DEVICE)
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind = case["kind"]
    return (_prepare_tables if kind == "tables" else _prepare_proj if kind == "proj" else _prepare_cache)(case, seed, gen)


# ---- one pass, in plain operations --------------------------------------------------------------------------------------
def _plain_append(st):
    k, v, slots, cache, scales = st["k"], st["v"], st["slots"], st["cache"], st["scales"]
    heads, D = k.shape[1], k.shape[2]
    blocks, run = torch.unique(slots // BLOCK, return_inverse=True)
    off = slots % BLOCK
    first = torch.full((blocks.numel(),), BLOCK, device=DEVICE).scatter_reduce(0, run, off, "amin")
    x = torch.stack([k, v], 2).float()                                                         # [tokens, heads, 2, D]
    top = torch.zeros((blocks.numel(), heads, 2), device=DEVICE).index_reduce(0, run, x.abs().amax(-1), "amax")
    want, had = _scale_of(top), scales[blocks]
    now = torch.where((first > 0)[:, None, None], torch.maximum(had, want), want)
    page = cache[blocks].view(FP8).view(blocks.numel(), heads, 2, BLOCK * D).float()
    page = torch.stack([page[:, :, 0].view(-1, heads, BLOCK, D), page[:, :, 1].view(-1, heads, D, BLOCK).transpose(2, 3)], 2)
    front = (torch.arange(BLOCK, device=DEVICE) < first[:, None])[:, None, None, :, None]
    page = torch.where(front, page * (had / now)[..., None, None], page)
    page[run, :, :, off] = x / now[run][..., None]
    page = _codes(page)
    cache[blocks, :, 0] = page[:, :, 0].reshape(-1, heads, BLOCK * D)
    cache[blocks, :, 1] = page[:, :, 1].transpose(2, 3).reshape(-1, heads, BLOCK * D)
    scales[blocks] = now


def _plain_attend(st, q, cu, seqs, max_q, max_len, out):
    """Rows q of the sequences in the slice `seqs`, their lengths in rows from cu, against what the cache stands for."""
    heads, D = st["cache"].shape[1], q.shape[2]
    lens, nb = st["seq_lens"][seqs].long(), _blocks(max_len)
    pages = st["table"][seqs, :nb].long().clamp(min=0)
    S, G, M = pages.shape[0], q.shape[1] // heads, nb * BLOCK
    codes, scale = st["cache"][pages].view(FP8).float(), st["scales"][pages][..., None]             # [S, nb, heads, 2, BLOCK * D]
    codes = codes * scale
    k = codes[..., 0, :].view(S, nb, heads, BLOCK, D).transpose(1, 2).reshape(S, heads, M, D)
    v = codes[..., 1, :].view(S, nb, heads, D, BLOCK).permute(0, 2, 1, 4, 3).reshape(S, heads, M, D)
    del codes
    n = cu[1:] - cu[:-1]
    i = torch.arange(max_q, device=DEVICE)
    row = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1)                                            # [S, max_q]
    pos = (lens - n)[:, None] + i
    qs = q[row].float().view(S, max_q, heads, G, D).permute(0, 2, 3, 1, 4).reshape(S, heads, G * max_q, D)
    logits = torch.matmul(qs, k.transpose(2, 3).contiguous()).mul_(st["scale"]).view(S, heads, G, max_q, M)
    hidden = torch.arange(M, device=DEVICE) > torch.minimum(pos, lens[:, None] - 1)[..., None]      # [S, max_q, M]
    logits.masked_fill_(hidden[:, None, None], float("-inf"))
    logits.sub_(logits.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(logits.view(S, heads, G * max_q, M), v).view(S, heads, G, max_q, D) / logits.sum(-1, keepdim=True)
    there = i < n[:, None]
    out[row[there]] = o.permute(0, 3, 1, 2, 4).reshape(S, max_q, heads * G, D)[there].to(out.dtype)


def _plain_tables(st):
    new, lens, table, free, count = st["new"].long().clamp(min=0), st["lens"].long().clamp(min=0), st["table"], st["free"], st["count"]
    seqs, wide = table.shape
    i = torch.arange(seqs, device=DEVICE)
    chunk = i < st["n_pre"]
    ok = (lens + new <= wide * BLOCK) & (chunk | (new <= 1))
    asked = torch.where(chunk & ok, new, 0).cumsum(0)
    ok &= ~chunk | (asked <= st["q_rows"])
    had, then = (lens + BLOCK - 1) // BLOCK, (lens + new + BLOCK - 1) // BLOCK
    need = torch.where(ok, then - had, 0)
    ok &= (need == 0) | (need.cumsum(0) <= count)
    taken, need = torch.where(ok, new, 0), torch.where(ok, need, 0)
    # blocks from the top of the stack
    col = torch.arange(wide, device=DEVICE)
    at = count - 1 - (need.cumsum(0) - need)[:, None] - (col - had[:, None])
    fresh = (col >= had[:, None]) & (col < (had + need)[:, None])
    table.copy_(torch.where(fresh, free[at.clamp(0, free.numel() - 1).long()], table))
    left = count - need.sum()
    # rows of the chunks one behind the other, then one row for each decode sequence
    starts = torch.where(chunk, taken, 0).cumsum(0)
    cu = torch.cat([starts.new_zeros(1), starts[:st["n_pre"]]])
    r = torch.arange(st["slots"].numel(), device=DEVICE)
    in_chunks = r < st["q_rows"]
    s = torch.where(in_chunks, torch.searchsorted(cu, r, right=True) - 1, r - st["q_rows"] + st["n_pre"])
    used = torch.where(in_chunks, s < st["n_pre"], s < seqs)
    s = s.clamp(0, seqs - 1)
    used &= taken[s] > 0
    first = torch.cat([cu[:-1], torch.arange(seqs - st["n_pre"], device=DEVICE) + st["q_rows"]])
    p = (lens[s] + r - first[s]).clamp(0, wide * BLOCK - 1)
    st["slots"].copy_(torch.where(used, table[s, p // BLOCK].long() * BLOCK + p % BLOCK, -1))
    st["cu"].copy_(cu)
    st["taken"].copy_(taken)
    st["lens"].copy_(lens + taken)
    count.copy_(left)
    # the same tokens given back
    now, keep = st["lens"].long(), st["before"].long()
    keep = torch.where((keep < 0) | (keep > now), now, keep)
    kept, back = (keep + BLOCK - 1) // BLOCK, (now + BLOCK - 1) // BLOCK
    gone = back - kept
    total = gone.sum()
    at = count + total - 1 - (gone.cumsum(0) - gone)[:, None] - (col - kept[:, None])
    put = (col >= kept[:, None]) & (col < back[:, None])
    free[at[put]] = table[put]
    count.add_(total)
    st["lens"].copy_(keep)


def _plain_proj(st):
    P, h, h_kv = st["P"], st["h"], st["h_kv"]
    T = st["x"].shape[0]
    xc, xs = _quantise_rows(st["x"])
    st["xc"].copy_(xc)
    st["xs"].copy_(xs)
    y = torch.matmul(xc.float(), st["w_qkv"].float().t()).mul_(xs[:, None]).mul_(st["ws_qkv"]).to(torch.bfloat16).view(T, h + 2 * h_kv, 128)
    hq, hkv = h // P, _kv_heads_here(P, h_kv)
    dest = torch.arange(P, device=DEVICE)[:, None]
    kv = dest * h_kv // P + torch.arange(hkv, device=DEVICE)
    heads = torch.cat([dest * hq + torch.arange(hq, device=DEVICE), h + kv, h + h_kv + kv], 1)       # [P, hq + 2 hkv]
    st["send"][:, :T] = y[:, heads].transpose(0, 1)
    st["send"][:, T:] = 0
    rows = st["recv"][:, :T].transpose(0, 1).reshape(T, h * 128)
    rc, rs = _quantise_rows(rows)
    st["rc"][:, :T] = rc.view(T, P, hq, 128).transpose(0, 1)
    st["rs"].copy_(rs)
    st["out"].copy_(torch.matmul(rc.float(), st["w_o"].float().t()).mul_(rs[:, None]).mul_(st["ws_o"]))


# ---- one pass, through the framework's operators ------------------------------------------------------------------------
def _workspace(need):
    return torch.empty(max(need, 16), dtype=torch.uint8, device=DEVICE)


def _own_pass(st):
    from paper_2509_16495_amd import binding as B
    kind = st["kind"]
    if kind == "tables":
        if st["ws"] is None:
            st["ws"] = _workspace(B.tables_workspace_bytes(st["new"].numel()))
        B.tables_append(st["new"], st["n_pre"], st["q_rows"], st["lens"], st["table"], st["free"], st["count"], st["cu"], st["slots"], st["taken"],
                        workspace=st["ws"])
        B.tables_truncate(st["before"], st["lens"], st["table"], st["free"], st["count"], workspace=st["ws"])
        return
    if kind == "proj":
        if st["ws"] is None:
            rows, n, d, k = st["send"].shape[1], st["w_qkv"].shape[0], st["w_qkv"].shape[1], st["w_o"].shape[1]
            st["ws"] = _workspace(max(B.proj_workspace_bytes_int8(rows, n, d), B.proj_workspace_bytes_int8(st["x"].shape[0], d, k)))
        B.quantize_rows_int8(st["x"], st["xc"], st["xs"])
        B.qkv_proj_pack_int8(st["xc"], st["xs"], st["w_qkv"], st["ws_qkv"], st["send"], st["P"], st["h"], st["h_kv"], workspace=st["ws"])
        B.quantize_recv_int8(st["recv"], st["rc"], st["rs"])
        B.unpack_o_proj_int8(st["rc"], st["rs"], st["w_o"], st["ws_o"], st["out"], workspace=st["ws"])
        return
    if kind == "append":
        B.kv_write(st["k"], st["v"], st["slots"], st["cache"], kv_scales=st["scales"])
        return
    seqs = st["seq_lens"].numel()
    if st["ws"] is None:
        a = B.attn_desc(st["q"], st["cache"], st["table"], st["scale"], st["k"], st["out"], kv_scales=st["scales"])
        st["ws"] = _workspace(B.decode_workspace_bytes(seqs, st["max_dec"], a) if kind == "decode" else
                              B.prefill_workspace_bytes(seqs, st["q_rows"], st["max_q"], st["max_pre"], a) if kind == "prefill" else
                              B.mixed_workspace_bytes(st["n_pre"], st["q_rows"], st["max_q"], st["max_pre"], st["num_dec"], st["max_dec"], a))
    new = dict(k_new=st["k"], v_new=st["v"], slot_mapping=st["slots"], workspace=st["ws"], kv_scales=st["scales"])
    if kind == "decode":
        B.decode(st["q"], st["cache"], st["table"], st["seq_lens"], st["max_dec"], st["out"], st["scale"], **new)
    elif kind == "prefill":
        B.prefill(st["q"], st["cache"], st["table"], st["cu"], st["seq_lens"], st["max_q"], st["max_pre"], st["out"], st["scale"], **new)
    else:
        B.mixed(st["q"], st["cache"], st["table"], st["cu"], st["seq_lens"], st["n_pre"], st["max_q"], st["max_pre"], st["max_dec"], st["out"],
                st["scale"], **new)


def _plain_pass(st):
    kind = st["kind"]
    if kind == "tables":
        return _plain_tables(st)
    if kind == "proj":
        return _plain_proj(st)
    _plain_append(st)
    if kind == "append":
        return
    if st["n_pre"]:
        _plain_attend(st, st["q"], st["cu"].long(), slice(0, st["n_pre"]), st["max_q"], st["max_pre"], st["out"])
    if st["num_dec"]:
        at = st["q_rows"]
        _plain_attend(st, st["q"][at:], torch.arange(st["num_dec"] + 1, device=DEVICE), slice(st["n_pre"], None), 1, st["max_dec"], st["out"][at:])


def run(state):
    st = state
    if own:
        _own_pass(st)
    else:
        _plain_pass(st)
    if st["kind"] == "tables":
        return {"cu": st["cu"], "slots": st["slots"], "taken": st["taken"], "table": st["table"], "free": st["free"], "count": st["count"], "lens": st["lens"]}
    if st["kind"] == "proj":
        return {"x_codes": st["xc"], "x_scales": st["xs"], "send": st["send"], "recv_codes": st["rc"], "recv_scales": st["rs"], "out": st["out"]}
    res = {"cache": st["cache"].view(FP8), "scales": st["scales"]}
    if "out" in st:
        res["out"] = st["out"]
    return res


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------
def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_e4m3(x):
    """Nearest E4M3 value of doubles, ties to the even code: 2^(e - 3) apart in [2^e, 2^(e + 1)), 2^-9 below 2^-6."""
    e = (torch.frexp(x)[1] - 1).clamp(min=-6)
    step = _exact_power(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_scale(top):
    m, e = torch.frexp(top)   # top = m 2^e, 448 = 0.875 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    return _exact_power(torch.where(top == 0, E_MIN, e).clamp(E_MIN, E_MAX))


def _exact_pages(st, blocks):
    """Values of cache blocks as [blocks, heads, 2, BLOCK, D] doubles (codes, without the scales)."""
    c = torch.arange(256, device=DEVICE)
    m, e, sign = (c & 7).double(), (c >> 3) & 15, 1.0 - 2.0 * (c >> 7)
    value = sign * torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * _exact_power(e - 7))
    raw = value[st["cache"][blocks].int()]
    n, h, _, size = raw.shape
    D = size // BLOCK
    return torch.stack([raw[:, :, 0].reshape(n, h, BLOCK, D), raw[:, :, 1].reshape(n, h, D, BLOCK).transpose(2, 3)], 2)


def _exact_cache(case, st):
    """The cache's codes (as values) and scales behind the append, sequence by sequence; and each sequence's K and V."""
    codes, scales, per_seq, at = _exact_pages(st, torch.arange(st["cache"].shape[0], device=DEVICE)), st["scales"].double(), [], 0
    D = codes.shape[-1]
    for s, (n, c) in enumerate(_lengths(case)):
        b0 = (c - n) // BLOCK                        # the first block that gets new tokens
        ids = st["table"][s, b0:_blocks(c)].long()
        offset = c - n - b0 * BLOCK
        x = torch.zeros((codes.shape[1], 2, ids.numel() * BLOCK, D), dtype=torch.float64, device=DEVICE)
        x[:, 0, offset:offset + n] = st["k"][at:at + n].double().transpose(0, 1)
        x[:, 1, offset:offset + n] = st["v"][at:at + n].double().transpose(0, 1)
        x = x.view(codes.shape[1], 2, ids.numel(), BLOCK, D).permute(2, 0, 1, 3, 4).contiguous()
        now = _exact_scale(x.abs().amax((3, 4)))
        y = _exact_e4m3(x / now[..., None, None])
        if offset:
            now[0] = torch.maximum(now[0], scales[ids[0]])
            y[0] = _exact_e4m3(x[0] / now[0][..., None, None])
            y[0, :, :, :offset] = _exact_e4m3(codes[ids[0], :, :, :offset] * (scales[ids[0]] / now[0])[..., None, None])
        scales[ids] = now
        rows = torch.arange(ids.numel() * BLOCK, device=DEVICE).view(-1, BLOCK) < offset + n
        codes[ids] = torch.where(rows[:, None, None, :, None], y, codes[ids])
        at += n
    return codes, scales


def exact(case, seed):
    kind = case["kind"]
    if kind == "tables":
        return None   # whole numbers throughout
    st = prepare(case, seed)
    if kind == "proj":
        P, h, h_kv, T = st["P"], st["h"], st["h_kv"], case["T"]
        send = torch.zeros(st["send"].shape, dtype=torch.float64, device=DEVICE)
        hq, hkv = h // P, _kv_heads_here(P, h_kv)

        def product(x, w, ws):   # (bf16 activations, in 32 bits their scale and factor)
            top = x.abs().max(1).values.float()
            xs = (top / 127).double()
            codes = torch.round(x.double() * (127 / top).double()[:, None])
            return xs, codes, (codes @ w.double().t().contiguous()) * xs[:, None] * ws.double()
        xs, _, y = product(st["x"], st["w_qkv"], st["ws_qkv"])
        y = y.view(T, h + 2 * h_kv, 128)
        for p in range(P):
            g = p * h_kv // P
            send[p, :T, :hq] = y[:, p * hq:(p + 1) * hq]
            send[p, :T, hq:hq + hkv] = y[:, h + g:h + g + hkv]
            send[p, :T, hq + hkv:] = y[:, h + h_kv + g:h + h_kv + g + hkv]
        rs, _, out = product(torch.cat([st["recv"][p, :T].reshape(T, -1) for p in range(P)], 1), st["w_o"], st["ws_o"])
        return {"x_codes": None, "x_scales": xs, "send": send, "recv_codes": None, "recv_scales": rs, "out": out}
    codes, scales = _exact_cache(case, st)
    res = {"scales": scales}
    stored = codes.new_empty((codes.shape[0], codes.shape[1], 2, BLOCK * case["D"]))
    stored[:, :, 0] = codes[:, :, 0].reshape(codes.shape[0], codes.shape[1], -1)
    stored[:, :, 1] = codes[:, :, 1].transpose(2, 3).reshape(codes.shape[0], codes.shape[1], -1)
    res["cache"] = stored
    if kind == "append":
        return res
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEVICE)
    G, at = case["hq"] // case["hkv"], 0
    for s, (n, c) in enumerate(_lengths(case)):
        ids = st["table"][s, :_blocks(c)].long()
        kv = (codes[ids] * scales[ids][..., None, None]).permute(1, 2, 0, 3, 4).reshape(case["hkv"], 2, -1, case["D"])[:, :, :c]
        later = torch.arange(c, device=DEVICE) > torch.arange(c - n, c, device=DEVICE)[:, None]
        for j in range(case["hq"]):
            logits = (st["q"][at:at + n, j].double() @ kv[j // G, 0].t().contiguous()) * st["scale"]
            out[at:at + n, j] = torch.softmax(logits.masked_fill_(later, -math.inf), -1) @ kv[j // G, 1]
        at += n
    res["out"] = out
    return res
