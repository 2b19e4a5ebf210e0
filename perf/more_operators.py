"""What is measured of the operators around a layer's projections and of decoding behind a shared prompt: the residual addition with its
root-mean-square norm (in 16, 32 or 8 bits), rotary positions, and decode attention whose groups of sequences share the first blocks of
their tables.

`listed()` names eleven cases and `draw()` picks more from the same ranges; `prepare()` makes what a serving program holds before the
call, `run()` is one pass: in plain torch operations, or, where `own` is true, through `paper_2509_16495_amd.binding`.  A case is a
dict of plain values; its `kind` says which operator it takes:

  norm     x added to the residual stream in place, its norm times a weight, written as values or as 8-bit codes with a scale per row
  rotary   query and key heads of fused q|k|v rows turned by their positions, in place
  shared   one new token per sequence, with its append, over a paged cache in which groups of sequences have a prefix in common

Head geometries are those of the models the repository serves (64q/8kv, 40q/8kv, 32q/8kv, 32q/4kv, head_dim 128) split over GPUs, row
lengths their d_model.  Lengths come from the case's own `lens_seed`, so every preparation of a case has the same amount of work; values
and block tables come from the preparation's seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16
DEVICE = "cuda:0"
FP8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.uint8, "int8": torch.int8}
EPS = 1e-5

D_MODELS = (2048, 4096, 5120, 8192)
GPU_HEADS = ((8, 1), (8, 1), (4, 1), (5, 1), (16, 2), (10, 2))   # (query, KV) heads on one GPU


def listed():
    return [
        # one sequence decodes: a single row, latency counts
        dict(name="norm_1_row", kind="norm", rows=1, cols=8192, x="bf16", res="bf16", out="bf16", offset=0.0),
        # a decode step's rows, straight into what the int8 projections take
        dict(name="norm_19_rows_int8", kind="norm", rows=19, cols=8192, x="bf16", res="bf16", out="int8", offset=0.0),
        # a ragged chunked-prefill step over FP8 projections, the residual stream kept in 32 bits
        dict(name="norm_2041_rows_fp8", kind="norm", rows=2041, cols=5120, x="bf16", res="f32", out="fp8", offset=0.0),
        # a large prefill
        dict(name="norm_16384_rows_int8", kind="norm", rows=16384, cols=8192, x="bf16", res="bf16", out="int8", offset=0.0),
        # rows of a decode step far into their contexts
        dict(name="rotary_decode_97", kind="rotary", mixed=False, chunks=0, len_lo=0, len_hi=0, cached=0, decs=97, ctx_lo=1000, ctx_hi=131072, hq=8, hkv=1, D=128,
             rot=128, pairs=False, dtype="bf16", lens_seed=11),
        # one unified step: prompts, chunks behind cached tokens and decode rows, positions from the lengths that the attention call takes
        dict(name="rotary_mixed_step", kind="rotary", mixed=True, chunks=5, len_lo=1, len_hi=6000, cached=20000, decs=200, ctx_lo=1, ctx_hi=16000, hq=16, hkv=2,
             D=128, rot=64, pairs=True, dtype="bf16", lens_seed=12),
        # the rows of a long prompt in TP mode, two KV heads a GPU
        dict(name="rotary_prompt_65536", kind="rotary", mixed=True, chunks=1, len_lo=65536, len_hi=65536, cached=0, decs=0, ctx_lo=0, ctx_hi=0, hq=16, hkv=2, D=128,
             rot=128, pairs=False, dtype="bf16", lens_seed=13),
        # four answers sampled from one prompt: latency counts
        dict(name="shared_4_answers", kind="shared", groups=1, size_lo=4, size_hi=4, pre_lo=4000, pre_hi=4100, suf_lo=1, suf_hi=300, alone=0, alone_hi=0, hq=8, hkv=1,
             cache="bf16", lens_seed=14),
        # a serving batch behind one long system prompt, conversations of different length, a few others among them
        dict(name="shared_64_chats", kind="shared", groups=1, size_lo=61, size_hi=61, pre_lo=16391, pre_hi=16391, suf_lo=1, suf_hi=1500, alone=3, alone_hi=9000, hq=8,
             hkv=1, cache="bf16", lens_seed=15),
        # several documents, each questioned by many sequences, FP8 cache
        dict(name="shared_8_documents_fp8", kind="shared", groups=8, size_lo=5, size_hi=40, pre_lo=3000, pre_hi=30000, suf_lo=1, suf_hi=800, alone=9, alone_hi=5000, hq=8,
             hkv=1, cache="fp8", lens_seed=16),
        # the largest: 256 sequences behind one prompt, where the shared part is bound by matrix products
        dict(name="shared_256_seqs", kind="shared", groups=1, size_lo=256, size_hi=256, pre_lo=32768, pre_hi=32768, suf_lo=200, suf_hi=2000, alone=0, alone_hi=0, hq=8,
             hkv=1, cache="bf16", lens_seed=17),
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "rotary", "rotary", "shared", "shared", "shared"])
    seed = rng.randrange(1 << 30)
    if kind == "norm":
        cols = rng.choice([rng.choice(D_MODELS), rng.choice(D_MODELS), 8 * _log_int(rng, 8, 2048)])
        return dict(kind=kind, rows=_log_int(rng, 1, min(16384, (1 << 27) // cols)), cols=cols, x=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                    res=rng.choice(["bf16", "bf16", "f32", "none"]), out=rng.choice(["bf16", "fp8", "int8", "int8", "f32"]), offset=rng.choice([0.0, 0.0, 1.0]))
    if kind == "rotary":
        chunks, hi = rng.choice([0, _log_int(rng, 1, 30)]), _log_int(rng, 20, 9000)
        decs = _log_int(rng, 1, 300) if chunks == 0 else rng.choice([0, _log_int(rng, 1, 300)])
        hq, hkv = rng.choice(GPU_HEADS)
        D = rng.choice([128, 128, 128, 64])
        return dict(kind=kind, mixed=rng.choice([True, False]), chunks=min(chunks, max(1, 60000 // hi)) if chunks else 0, len_lo=1, len_hi=hi,
                    cached=rng.choice([0, 0, _log_int(rng, 10, 100000)]), decs=decs, ctx_lo=1, ctx_hi=_log_int(rng, 40, 131072), hq=hq, hkv=hkv, D=D,
                    rot=rng.choice([D, D, D // 2, D // 4]), pairs=rng.choice([False, False, True]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), lens_seed=seed)
    hq, hkv = rng.choice(GPU_HEADS)
    seqs = _log_int(rng, 2, 256)
    groups = min(_log_int(rng, 1, 12), max(1, seqs // 2))
    pre = _log_int(rng, 40, min(32768, 60_000_000 // (seqs * hq)))
    suf = _log_int(rng, 2, 2000)
    alone = rng.choice([0, 0, _log_int(rng, 1, 20)])
    size = max(2, seqs // groups)
    return dict(kind=kind, groups=groups, size_lo=max(1, size // 2), size_hi=size, pre_lo=max(1, pre // rng.choice([1, 2, 8])), pre_hi=pre, suf_lo=1, suf_hi=suf,
                alone=alone, alone_hi=_log_int(rng, 16, 9000) if alone else 0, hq=hq, hkv=hkv, cache=rng.choice(["bf16", "bf16", "fp8"]), lens_seed=seed)


# ---- sizes of a case ---------------------------------------------------------------------------------------------------
def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _lengths(case):
    """(new tokens, tokens with them) per sequence: chunks and prompts first, then decode rows."""
    r = random.Random(case["lens_seed"])
    lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["chunks"])]
    return ([(n, n + (case["cached"] if i % 2 else 0)) for i, n in enumerate(lens)] + [(1, r.randint(case["ctx_lo"], case["ctx_hi"])) for _ in range(case["decs"])])


def _families(case):
    """Tokens in common and the sequences' lengths, group by group; then the lengths of the sequences of no group."""
    r = random.Random(case["lens_seed"])
    groups = []
    for _ in range(case["groups"]):
        pre = r.randint(case["pre_lo"], case["pre_hi"])
        groups.append((pre, [pre + r.randint(case["suf_lo"], case["suf_hi"]) for _ in range(r.randint(case["size_lo"], case["size_hi"]))]))
    return groups, [r.randint(1, case["alone_hi"]) for _ in range(case["alone"])]


def work(case):
    kind = case["kind"]
    size = {"bf16": 2, "f32": 4, "fp8": 1, "int8": 1, "none": 0}
    if kind == "norm":
        n, rows = case["cols"], case["rows"]
        return {"bytes": rows * n * (size[case["x"]] + 2 * size[case["res"]] + size[case["out"]]) + 2 * n + (4 * rows if case["out"] in ("fp8", "int8") else 0),
                "flops": 5 * rows * n}
    if kind == "rotary":
        lens = _lengths(case)
        rows = sum(n for n, _ in lens)
        return {"bytes": rows * (case["hq"] + case["hkv"]) * case["rot"] * 2 * size[case["dtype"]] + 4 * case["rot"] + (8 * len(lens) if case["mixed"] else 4 * rows),
                "flops": 3 * rows * (case["hq"] + case["hkv"]) * case["rot"]}
    groups, alone = _families(case)
    e, hq, hkv, D = size[case["cache"]], case["hq"], case["hkv"], 128
    lens = [c for _, m in groups for c in m] + alone
    once = sum(pre // BLOCK * BLOCK + sum(c - pre // BLOCK * BLOCK for c in m) for pre, m in groups) + sum(alone)
    return {"bytes": (once - len(lens)) * 2 * hkv * D * e + len(lens) * (2 * hq * D * 2 + 2 * hkv * D * (2 + e) + 12), "flops": 4 * D * hq * sum(lens)}


# ---- preparation -------------------------------------------------------------------------------------------------------
def _normal(shape, dtype, gen, std=1.0):
    return torch.empty(shape, dtype=dtype, device=DEVICE).normal_(0.0, std, generator=gen)


def _prepare_norm(case, seed, gen):
    rows, cols = case["rows"], case["cols"]
    # tokens of different magnitude, a few channels that stand out, as in a trained model's residual stream
    loud = torch.ones(cols, device=DEVICE)
    loud[torch.randperm(cols, generator=gen, device=DEVICE)[:max(1, cols // 512)]] = 20.0
    st = {"kind": "norm", "offset": case["offset"], "out_kind": case["out"]}
    st["x"] = _normal((rows, cols), torch.float32, gen).mul_(_normal((rows, 1), torch.float32, gen, 0.5).exp_()).to(TYPES[case["x"]])
    st["res"] = None if case["res"] == "none" else _normal((rows, cols), torch.float32, gen, 3.0).mul_(loud).to(TYPES[case["res"]])
    st["w"] = (_normal((cols,), torch.float32, gen, 0.2) + (1.0 - case["offset"])).to(torch.bfloat16)
    st["out"] = torch.empty((rows, cols), dtype=TYPES[case["out"]], device=DEVICE)
    st["scales"] = torch.empty(rows, dtype=torch.float32, device=DEVICE) if case["out"] in ("fp8", "int8") else None
    return st


def _prepare_rotary(case, seed, gen):
    lens = _lengths(case)
    hq, hkv, D, half = case["hq"], case["hkv"], case["D"], case["rot"] // 2
    new, total = torch.tensor([n for n, _ in lens], device=DEVICE), torch.tensor([c for _, c in lens], device=DEVICE)
    rows = int(new.sum())
    buf = _normal((rows, hq + 2 * hkv, D), torch.float32, gen).to(TYPES[case["dtype"]])   # the fused rows that the exchange delivers
    st = {"kind": "rotary", "mixed": case["mixed"], "buf": buf, "q": buf[:, :hq], "k": buf[:, hq:hq + hkv], "rot": case["rot"], "pairs": case["pairs"],
          "n_pre": case["chunks"], "q_rows": sum(n for n, _ in lens[:case["chunks"]]), "seq_lens": total.to(torch.int32)}
    st["freq"] = torch.exp(torch.arange(half, dtype=torch.float64, device=DEVICE) * (-math.log(500000.0) / half))
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    st["cu"] = cu[:case["chunks"] + 1].to(torch.int32)
    s = torch.repeat_interleave(torch.arange(len(lens), device=DEVICE), new)
    st["pos"] = (torch.arange(rows, device=DEVICE) - cu[s] + (total - new)[s]).to(torch.int32)
    return st


def _prepare_shared(case, seed, gen):
    groups, alone = _families(case)
    hq, hkv, D = case["hq"], case["hkv"], 128
    lens = torch.tensor([c for _, m in groups for c in m] + alone, device=DEVICE)
    sizes = [len(m) for _, m in groups]
    pre = torch.tensor([p for p, _ in groups], device=DEVICE)
    grouped = torch.repeat_interleave(torch.arange(len(groups), device=DEVICE), torch.tensor(sizes, device=DEVICE))
    common = torch.zeros_like(lens)                                      # blocks in common, per sequence
    common[:grouped.numel()] = pre[grouped] // BLOCK
    wide = int(((lens + BLOCK - 1) // BLOCK).max())
    own_blocks = (lens + BLOCK - 1) // BLOCK - common
    shared_blocks = pre // BLOCK
    used = int(own_blocks.sum() + shared_blocks.sum())
    num_blocks = used + used // 8 + 1
    order = torch.randperm(num_blocks, generator=gen, device=DEVICE).to(torch.int32)
    i = torch.arange(wide, device=DEVICE)
    at = (own_blocks.cumsum(0) - own_blocks)[:, None] + int(shared_blocks.sum()) + i - common[:, None]
    table = torch.where(i < (common + own_blocks)[:, None], order[at.clamp(0, num_blocks - 1)], -1)
    first = torch.zeros_like(lens)
    first[:grouped.numel()] = (shared_blocks.cumsum(0) - shared_blocks)[grouped]
    table = torch.where(i < common[:, None], order[(first[:, None] + i).clamp(max=num_blocks - 1)], table).contiguous()
    st = {"kind": "shared", "scale": 1.0 / math.sqrt(D), "table": table, "seq_lens": lens.to(torch.int32), "max_len": int(lens.max()), "ws": None,
          "fp8": case["cache"] == "fp8", "factors": (0.03, 0.02) if case["cache"] == "fp8" else (1.0, 1.0)}
    st["offsets"] = torch.tensor([sum(sizes[:j]) for j in range(len(sizes) + 1)], dtype=torch.int32, device=DEVICE)
    st["shared_lens"] = pre.to(torch.int32)
    last = lens - 1
    st["slots"] = table[torch.arange(lens.numel(), device=DEVICE), last // BLOCK].long() * BLOCK + last % BLOCK
    values = _normal((num_blocks, hkv, 2, BLOCK * D), torch.bfloat16, gen)
    if st["fp8"]:
        values[:, :, 0].div_(st["factors"][0])
        values[:, :, 1].div_(st["factors"][1])
        values = values.clamp_(-448.0, 448.0).to(FP8).view(torch.uint8)
    st["cache"] = values
    rows = _normal((lens.numel(), hq + 2 * hkv, D), torch.bfloat16, gen)   # the fused rows that the exchange delivers
    rows[:, :hq].mul_(2.0)
    st["q"], st["k"], st["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    st["out"] = torch.empty((lens.numel(), hq, D), dtype=torch.bfloat16, device=DEVICE)
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return {"norm": _prepare_norm, "rotary": _prepare_rotary, "shared": _prepare_shared}[case["kind"]](case, seed, gen)


# ---- one pass, in plain operations --------------------------------------------------------------------------------------
def _plain_norm(st):
    h = st["x"].float()
    if st["res"] is not None:
        st["res"].copy_(h + st["res"].float())
        h = st["res"].float()
    # the mean in 64 bits: codes are compared one by one, and its last bit of 32 would decide those next to a border
    inv = (h.double().square().mean(-1, keepdim=True) + EPS).rsqrt().float()
    y = h * inv * (st["w"].float() + st["offset"])
    if st["scales"] is None:
        st["out"].copy_(y)
        return
    top = y.abs().amax(-1, keepdim=True)
    if st["out_kind"] == "fp8":
        scale = torch.where(top > 0, top / 448.0, 1.0)
        st["out"].copy_((y / scale).clamp(-448.0, 448.0).to(FP8).view(torch.uint8))
    else:
        tiny = top < 2.0 ** -100
        scale = torch.where(tiny, 1.0, top * torch.tensor(1.0 / 127.0, dtype=torch.float32))
        inv = torch.where(tiny, 1.0, top.reciprocal() * 127.0)
        # the product of two float32 values is exact in 64 bits: nearest code, ties to the even one
        st["out"].copy_((y.double() * inv.double()).round_())
    st["scales"].copy_(scale.squeeze(-1))


def _plain_rotary(st):
    pos = st["pos"]
    if st["mixed"]:
        r = torch.arange(st["buf"].shape[0], device=DEVICE)
        chunk = r < st["q_rows"]
        s = torch.where(chunk, torch.searchsorted(st["cu"].long(), r, right=True) - 1, r - st["q_rows"] + st["n_pre"])
        ends = torch.cat([st["cu"][1:].long(), torch.arange(st["seq_lens"].numel() - st["n_pre"], device=DEVICE) + st["q_rows"] + 1])
        pos = st["seq_lens"].long()[s] - ends[s] + r
    angle = pos.double()[:, None] * st["freq"]      # far positions: 32 bits have no fraction of a turn left
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = st["rot"] // 2
    heads = st["buf"][:, :st["q"].shape[1] + st["k"].shape[1], :st["rot"]]
    x = heads.float()
    a, b = (x[..., 0::2], x[..., 1::2]) if st["pairs"] else (x[..., :half], x[..., half:])
    turned = (a * cos - b * sin, b * cos + a * sin)
    heads.copy_(torch.stack(turned, -1).flatten(-2) if st["pairs"] else torch.cat(turned, -1))


def _plain_shared(st):
    cache, slots, table = st["cache"], st["slots"], st["table"]
    hkv, D = cache.shape[1], st["q"].shape[2]
    blk, off = slots // BLOCK, slots % BLOCK
    for part, x in ((0, st["k"]), (1, st["v"])):
        if st["fp8"]:
            x = (x.float() / st["factors"][part]).clamp(-448.0, 448.0).to(FP8).view(torch.uint8)
        page = cache[:, :, part].view(-1, hkv, BLOCK, D) if part == 0 else cache[:, :, part].view(-1, hkv, D, BLOCK).transpose(2, 3)
        page[blk, :, off] = x
    pages = table.long().clamp(min=0)
    S, nb, G = table.shape[0], table.shape[1], st["q"].shape[1] // hkv
    M = nb * BLOCK
    gathered = cache[pages]                                                     # [S, nb, hkv, 2, BLOCK * D]
    if st["fp8"]:
        gathered = gathered.view(FP8)
    k = gathered[..., 0, :].float().view(S, nb, hkv, BLOCK, D).transpose(1, 2).reshape(S, hkv, M, D)
    q = st["q"].float().view(S, hkv, G, D)
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st["scale"] * st["factors"][0])
    del k
    there = torch.arange(M, device=DEVICE) < st["seq_lens"][:, None]
    logits.masked_fill_(~there[:, None, None], float("-inf"))
    logits.sub_(logits.amax(-1, keepdim=True)).exp_()
    v = gathered[..., 1, :].float().view(S, nb, hkv, D, BLOCK).permute(0, 2, 1, 4, 3).reshape(S, hkv, M, D)
    out = torch.matmul(logits, v) * st["factors"][1] / logits.sum(-1, keepdim=True)
    st["out"].copy_(out.view(S, hkv * G, D))


# ---- one pass, through the framework's operators ------------------------------------------------------------------------
def _own_pass(st):
    from paper_2509_16495_amd import binding as B
    if st["kind"] == "norm":
        B.add_rms_norm(st["x"], st["w"], st["out"], EPS, residual=st["res"], scales=st["scales"], weight_offset=st["offset"])
    elif st["kind"] == "rotary":
        if st["mixed"]:
            B.rotary_mixed(st["q"], st["k"], st["cu"], st["seq_lens"], st["n_pre"], st["freq"], pairs=st["pairs"])
        else:
            B.rotary(st["q"], st["k"], st["pos"], st["freq"], pairs=st["pairs"])
    else:
        if st["ws"] is None:
            a = B.attn_desc(st["q"], st["cache"], st["table"], st["scale"], st["k"], st["out"], *st["factors"])
            need = B.decode_shared_workspace_bytes(st["seq_lens"].numel(), st["max_len"], st["shared_lens"].numel(), a)
            st["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEVICE)
        B.decode_shared(st["q"], st["cache"], st["table"], st["seq_lens"], st["max_len"], st["offsets"], st["shared_lens"], st["out"], st["scale"],
                        k_new=st["k"], v_new=st["v"], slot_mapping=st["slots"], workspace=st["ws"], k_scale=st["factors"][0], v_scale=st["factors"][1])


def run(state):
    st = state
    if own:
        _own_pass(st)
    else:
        {"norm": _plain_norm, "rotary": _plain_rotary, "shared": _plain_shared}[st["kind"]](st)
    if st["kind"] == "norm":
        res = {"out": st["out"].view(FP8) if st["out_kind"] == "fp8" else st["out"]}
        if st["res"] is not None:
            res["residual"] = st["res"]
        if st["scales"] is not None:
            res["scales"] = st["scales"]
        return res
    if st["kind"] == "rotary":
        return {"rows": st["buf"]}
    return {"out": st["out"], "cache": st["cache"].view(FP8) if st["fp8"] else st["cache"]}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------
def _exact_e4m3(c):
    """Values of E4M3 codes."""
    n = torch.arange(256, device=DEVICE)
    m, e, sign = (n & 7).double(), (n >> 3) & 15, 1.0 - 2.0 * (n >> 7)
    value = sign * torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.ldexp(torch.ones_like(m), e - 7))
    return value[c.int()]


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "norm":
        h, res = st["x"].double(), {}
        if st["res"] is not None:
            res["residual"] = h + st["res"].double()
            h = res["residual"].to(st["res"].dtype).double()      # what the stream keeps is what is normalised
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["cols"] + EPS) * (st["w"].double() + case["offset"])
        if st["scales"] is None:
            return {**res, "out": y}
        scale = y.abs().amax(1, keepdim=True) / (448 if case["out"] == "fp8" else 127)
        return {**res, "scales": scale[:, 0], "out": y / scale if case["out"] == "fp8" else None}
    if case["kind"] == "rotary":
        rows, i = st["buf"].double(), 0
        heads, half = case["hq"] + case["hkv"], case["rot"] // 2
        lo = torch.arange(half, device=DEVICE) * (2 if case["pairs"] else 1)
        hi = lo + (1 if case["pairs"] else half)
        for n, c in _lengths(case):
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), torch.arange(c - n, c, device=DEVICE)[:, None, None] * st["freq"])
            z = torch.complex(rows[i:i + n, :heads][..., lo], rows[i:i + n, :heads][..., hi]) * turn
            rows[i:i + n, :heads, lo] = z.real
            rows[i:i + n, :heads, hi] = z.imag
            i += n
        return {"rows": rows}
    hkv, G, D = case["hkv"], case["hq"] // case["hkv"], 128
    out = torch.empty(st["out"].shape, dtype=torch.float64, device=DEVICE)
    for s, c in enumerate(st["seq_lens"].tolist()):
        ids = st["table"][s, :_blocks(c)].long()
        page = st["cache"][ids]
        page = _exact_e4m3(page) if st["fp8"] else page.double()
        for g in range(hkv):
            k = page[:, g, 0].reshape(-1, D)[:c] * st["factors"][0]
            v = page[:, g, 1].reshape(-1, D, BLOCK).transpose(1, 2).reshape(-1, D)[:c] * st["factors"][1]
            new_k, new_v = st["k"][s, g], st["v"][s, g]
            if st["fp8"]:   # the new token as the cache keeps it
                new_k, new_v = (_exact_e4m3((x.float() / f).clamp(-448.0, 448.0).to(FP8).view(torch.uint8)) * f for x, f in zip((new_k, new_v), st["factors"]))
            k[c - 1], v[c - 1] = new_k.double(), new_v.double()
            p = torch.softmax((st["q"][s, g * G:(g + 1) * G].double() @ k.t().contiguous()) * st["scale"], -1)
            out[s, g * G:(g + 1) * G] = p @ v
    return {"out": out, "cache": None}
