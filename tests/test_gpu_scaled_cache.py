"""The FP8 cache with a scale for each block and head: its append bit for bit, attention over it against 64 bits."""
import numpy as np
import pytest

import plain_8bit as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _rows(rng, n, heads, D, dtype):
    """Values of tokens of different magnitude."""
    x = (rng.standard_normal((n, heads, D)) * np.exp(rng.standard_normal((n, 1, 1)))).astype(np.float32)
    return P.bf16(x) if dtype == "bf16" else x


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.to(torch.bfloat16).cuda() if dtype == "bf16" else t.cuda()


class OnGpu:
    """A plain cache's codes and scales on the GPU."""

    def __init__(self, cache):
        self.codes, self.scales = _dev(cache.codes), _dev(cache.scales)

    def same(self, cache):
        got, want = self.codes.cpu().numpy(), cache.codes
        assert np.array_equal(self.scales.cpu().numpy(), cache.scales)
        assert np.array_equal(got, want), np.argwhere(got != want)[:5]


def _batch(rng, lens, heads, D, dtype, num_blocks=None):
    """A cache that holds the tokens in front of the new ones of sequences (new, total), filled in two calls, in blocks that others
    owned before; tables, slots of the new tokens and their K/V."""
    need = [-(-c // 16) for _, c in lens]
    num_blocks = num_blocks or sum(need) + 5
    cache, ids, at = P.Cache(num_blocks, heads, D, rng), rng.permutation(num_blocks), 0
    table = np.full((len(lens), max(need + [1])), -1, np.int32)
    slots = []
    for s, (n, c) in enumerate(lens):
        table[s, :need[s]] = ids[at:at + need[s]]
        at += need[s]
        sl = table[s, np.arange(c) // 16].astype(np.int64) * 16 + np.arange(c) % 16
        had = c - n
        for a, b in ((0, had // 2), (had // 2, had)):
            if b > a:
                x = _rows(rng, b - a, heads, 2 * D, dtype)
                cache.append(x[..., :D], x[..., D:], sl[a:b])
        slots.append(sl[had:])
    new = _rows(rng, sum(n for n, _ in lens), heads, 2 * D, dtype)
    return cache, table, np.concatenate(slots) if slots else np.zeros(0, np.int64), new[..., :D], new[..., D:]


SHAPES = [("bf16", 128, 1), ("bf16", 128, 3), ("bf16", 64, 2), ("f32", 64, 1), ("f32", 128, 2), ("bf16", 256, 1), ("bf16", 80, 1)]


@pytest.mark.parametrize("dtype,D,heads", SHAPES)
@pytest.mark.parametrize("lens", [
    [(1, 1)], [(1, 16), (1, 17), (1, 33), (1, 2)], [(16, 16)], [(40, 40), (7, 7), (100, 100)], [(37, 50), (3, 18), (1, 9), (200, 215), (1, 1), (5, 16)],
    [(1, 3 + 5 * i) for i in range(40)]])
def test_append_is_bit_exact(B, dtype, D, heads, lens):
    rng = np.random.Generator(np.random.PCG64(len(lens) + D))
    cache, table, slots, k, v = _batch(rng, lens, heads, D, dtype)
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    B.kv_write(_dev(k, dtype), _dev(v, dtype), _dev(slots), gpu.codes, kv_scales=gpu.scales)
    gpu.same(cache)


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("heads,lens", [(1, [(4200, 4205), (1, 1), (1, 90), (3, 3), (1, 17), (1, 18), (777, 800), (2, 33)]), (3, [(1500, 1500), (60, 71)] + [(1, 7 * i) for i in range(1, 40)])])
def test_append_of_many_tokens(B, heads, lens, D):
    """Batches in which a wavefront looks after several tokens: runs that cross its window, several of them in one, rows without a slot."""
    rng = np.random.Generator(np.random.PCG64(heads))
    cache, table, slots, k, v = _batch(rng, lens, heads, D, "bf16")
    pad = np.sort(rng.integers(0, len(lens), 3))            # in front of some sequences, so that the windows shift
    at = np.cumsum([0] + [n for n, _ in lens])[pad]
    slots, k, v = (np.insert(x, at, fill, 0) for x, fill in ((slots, -1), (k, 9.0), (v, 9.0)))
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    B.kv_write(_dev(k, "bf16"), _dev(v, "bf16"), _dev(slots), gpu.codes, kv_scales=gpu.scales)
    gpu.same(cache)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_a_block_filled_token_by_token(B, dtype, D):
    """Scales grow and stay as the largest token so far wants them; the codes in front follow."""
    rng = np.random.Generator(np.random.PCG64(5))
    cache, gpu = P.Cache(4, 2, D, rng), None
    gpu = OnGpu(cache)
    for t in range(37):
        x = _rows(rng, 1, 2, 2 * D, dtype) * np.float32(2.0 ** rng.integers(-12, 12))
        slots = np.array([[2, 0, 3][t // 16] * 16 + t % 16], np.int64)
        cache.append(x[..., :D], x[..., D:], slots)
        B.kv_write(_dev(x[..., :D], dtype), _dev(x[..., D:], dtype), _dev(slots), gpu.codes, kv_scales=gpu.scales)
        gpu.same(cache)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_append_of_values_at_the_edges(B, dtype, D):
    """Zeros, the smallest and largest numbers, infinities and NaN; padding rows in between; rows of a wider tensor; the top magnitudes at
    and next to 448 times a power of two."""
    rng = np.random.Generator(np.random.PCG64(6))
    k = _rows(rng, 64, 1, D, dtype)
    k[0] = 0
    k[1] = 1e-38
    k[2, 0, ::2], k[2, 0, 1::2] = -0.0, 3e38
    k[16:32] = 0
    k[32:48, 0, 3], k[33, 0, 5] = np.inf, np.nan
    k[40] = np.nan
    for i in range(16):
        k[48 + i] = np.float32(2.0 ** -20)
        k[48 + i, 0, i] = 448 * 2.0 ** -7 * (1 if i < 15 else 1 + 2.0 ** -7)
    k = P.bf16(k) if dtype == "bf16" else k
    v = np.ascontiguousarray(k[:, :, ::-1]) * np.float32(0.5)
    slots = np.r_[np.arange(16) + 32, np.arange(16) + 64, np.arange(16), np.arange(15) + 112, -1].astype(np.int64)
    cache = P.Cache(8, 1, D, rng)
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    wide = _dev(np.concatenate([v, k, k], 1), dtype)
    B.kv_write(wide[:, 2:], wide[:, :1], _dev(slots), gpu.codes, kv_scales=gpu.scales)
    got = gpu.codes.cpu().numpy()
    nan = (cache.codes & 0x7F) == 0x7F      # a NaN code of either sign
    assert np.array_equal(gpu.scales.cpu().numpy(), cache.scales) and np.array_equal(got[~nan], cache.codes[~nan]) and np.all((got[nan] & 0x7F) == 0x7F)


def test_every_code_moves_to_every_smaller_scale(B):
    """All 256 codes under ratios of 2^-1 .. 2^-18: exact, subnormal, rounded away."""
    rng = np.random.Generator(np.random.PCG64(7))
    for n in range(1, 19):
        cache = P.Cache(2, 1, 128, rng)
        cache.codes[1, 0, 0, :256] = cache.codes[1, 0, 1, ::16][:128].repeat(2) * 0 + np.arange(256)
        cache.codes[1, 0, 1].reshape(128, 16)[:, :2] = np.arange(256).reshape(128, 2)
        cache.scales[1] = 2.0 ** -3
        gpu = OnGpu(cache)
        x = np.full((1, 1, 128), 448 * 2.0 ** (n - 3), np.float32)
        cache.append(x, x, np.array([18]))
        B.kv_write(_dev(x, "bf16"), _dev(x, "bf16"), _dev(np.array([18])), gpu.codes, kv_scales=gpu.scales)
        got = gpu.codes.cpu().numpy()
        nan = (cache.codes & 0x7F) == 0x7F
        assert np.array_equal(got[~nan], cache.codes[~nan]) and np.all((got[nan] & 0x7F) == 0x7F)
        assert np.array_equal(gpu.scales.cpu().numpy(), cache.scales)




def _want(cache, table, lens, q):
    """Rows of all sequences one behind the other: result and bound's ingredients."""
    parts, at = [], 0
    D = q.shape[2]
    for s, (n, c) in enumerate(lens):
        parts.append(P.attend(q[at:at + n], cache, table[s], c, 1 / np.sqrt(D)) if c > 0 and n > 0 else tuple(np.zeros((n, q.shape[1], m)) for m in (D, D, 1)))
        at += n
    return [np.concatenate(x) for x in zip(*parts)]


def _check(got, want, dtype, D, keys):
    out, mag, big = want
    got = got.float().cpu().numpy().astype(np.float64)
    off = np.abs(got - out) / P.bound(dtype, out, mag, big, D, keys)
    assert np.all(np.isfinite(got)) and off.max() <= 1.0, (off.max(), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("dtype,D,hq,hkv", [("f32", 64, 9, 1), ("bf16", 48, 10, 2)])
def test_prefill_of_many_rows(B, dtype, D, hq, hkv):
    """Rows times heads beyond the line from which a workgroup takes several heads of a group (the last one fewer)."""
    _prefill(B, dtype, D, hq, hkv, [(900, 930), (61, 61)])


HEADS = [("bf16", 128, 8, 1), ("bf16", 128, 5, 1), ("bf16", 128, 10, 2), ("bf16", 128, 16, 1), ("bf16", 128, 40, 2), ("bf16", 64, 4, 1), ("f32", 64, 4, 2),
         ("f32", 128, 2, 1), ("bf16", 256, 2, 1)]


@pytest.mark.parametrize("dtype,D,hq,hkv", HEADS)
@pytest.mark.parametrize("lens", [[1], [1, 17, 250, 64, 33, 32, 16, 15, 1000], [700, 0, 2, 31, 0, 95], [40 + 7 * i for i in range(70)]])
@pytest.mark.parametrize("append", [True, False])
def test_decode(B, dtype, D, hq, hkv, lens, append):
    """Contexts of one token and many, padding rows (length 0), with the append in the call and in front of it."""
    import torch
    rng = np.random.Generator(np.random.PCG64(sum(lens) + D + hq))
    seqs = [(1 if c else 0, c) for c in lens]
    cache, table, slots, k, v = _batch(rng, seqs, hkv, D, dtype)
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    row = np.array([c > 0 for c in lens])
    kv = np.zeros((2, len(lens), hkv, D), np.float32)
    kv[:, row] = k, v
    sl = np.full(len(lens), -1, np.int64)
    sl[row] = slots
    q = _rows(rng, len(lens), hq, D, dtype)
    out = torch.full((len(lens), hq, D), np.nan, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    new = dict(k_new=_dev(kv[0], dtype), v_new=_dev(kv[1], dtype), slot_mapping=_dev(sl)) if append else {}
    if not append:
        B.kv_write(_dev(kv[0], dtype), _dev(kv[1], dtype), _dev(sl), gpu.codes, kv_scales=gpu.scales)
    B.decode(_dev(q, dtype), gpu.codes, _dev(table), _dev(np.array(lens, np.int32)), max(lens), out, 1 / np.sqrt(D), kv_scales=gpu.scales, **new)
    gpu.same(cache)
    want = _want(cache, table, [(1, c) for c in lens], q)
    _check(out, want, dtype, D, max(lens))
    assert not out.float().cpu().numpy()[~row].any()


@pytest.mark.parametrize("dtype,D,hq,hkv", HEADS)
@pytest.mark.parametrize("lens", [[(1, 1)], [(70, 70), (33, 200), (0, 5), (1, 1), (128, 300), (17, 40)], [(300, 311)]])
def test_prefill(B, dtype, D, hq, hkv, lens):
    _prefill(B, dtype, D, hq, hkv, lens)


def _prefill(B, dtype, D, hq, hkv, lens):
    import torch
    rng = np.random.Generator(np.random.PCG64(len(lens) * 31 + D + hq))
    cache, table, slots, k, v = _batch(rng, lens, hkv, D, dtype)
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    q = _rows(rng, len(slots), hq, D, dtype)
    fused = _dev(np.concatenate([q, k, v], 1), dtype)   # views into rows of q, k and v heads
    out = torch.empty((len(slots), hq, D), dtype=fused.dtype, device="cuda")
    cu = np.r_[0, np.cumsum([n for n, _ in lens])].astype(np.int32)
    B.prefill(fused[:, :hq], gpu.codes, _dev(table), _dev(cu), _dev(np.array([c for _, c in lens], np.int32)), max(n for n, _ in lens),
              max(c for _, c in lens), out, 1 / np.sqrt(D), k_new=fused[:, hq:hq + hkv], v_new=fused[:, hq + hkv:], slot_mapping=_dev(slots),
              kv_scales=gpu.scales)
    gpu.same(cache)
    _check(out, _want(cache, table, lens, q), dtype, D, max(c for _, c in lens))


@pytest.mark.parametrize("dtype,D,hq,hkv", [("bf16", 128, 8, 1), ("bf16", 128, 4, 2), ("f32", 64, 4, 1)])
@pytest.mark.parametrize("chunks,rows", [([(70, 70), (33, 200)], [1, 17, 250, 64, 0]), ([(150, 900)], [300 + 40 * i for i in range(24)]), ([], [5, 40]), ([(20, 25)], [])])
def test_mixed(B, dtype, D, hq, hkv, chunks, rows):
    import torch
    rng = np.random.Generator(np.random.PCG64(len(rows) + D + hq))
    lens = chunks + [(1 if c else 0, c) for c in rows]
    cache, table, slots, k, v = _batch(rng, lens, hkv, D, dtype)
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    n_chunk, total = sum(n for n, _ in chunks), sum(n for n, _ in chunks) + len(rows)
    there = np.r_[np.ones(n_chunk, bool), np.array([c > 0 for c in rows], bool)]
    kv, sl = np.zeros((2, total, hkv, D), np.float32), np.full(total, -1, np.int64)
    kv[:, there], sl[there] = (k, v), slots
    q = _rows(rng, total, hq, D, dtype)
    out = torch.empty((total, hq, D), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    cu = np.r_[0, np.cumsum([n for n, _ in chunks])].astype(np.int32)
    B.mixed(_dev(q, dtype), gpu.codes, _dev(table), _dev(cu), _dev(np.array([c for _, c in lens], np.int32)), len(chunks), max([n for n, _ in chunks], default=0),
            max([c for _, c in chunks], default=0), max(rows, default=0), out, 1 / np.sqrt(D), k_new=_dev(kv[0], dtype), v_new=_dev(kv[1], dtype),
            slot_mapping=_dev(sl), kv_scales=gpu.scales)
    gpu.same(cache)
    _check(out, _want(cache, table, chunks + [(1, c) for c in rows], q), dtype, D, max(c for _, c in lens))


def test_decode_steps_replayed_from_a_graph(B):
    """Blocks fill and scales grow from replay to replay, every step checked; two graphs share the workspace and run in turn."""
    import torch
    rng = np.random.Generator(np.random.PCG64(11))
    D, hq, hkv, start = 128, 8, 1, np.array([1, 14, 31, 100, 15])
    n, wide = len(start), 12
    cache = P.Cache(n * wide, hkv, D, rng)
    table = rng.permutation(n * wide).astype(np.int32).reshape(n, wide)
    slot_of = lambda s, p: int(table[s, p // 16]) * 16 + p % 16
    for s in range(n):
        x = _rows(rng, int(start[s]), hkv, 2 * D, "bf16")
        cache.append(x[..., :D], x[..., D:], np.array([slot_of(s, p) for p in range(start[s])]))
    gpu, tab = OnGpu(cache), _dev(table)
    lens, slots = _dev(start.astype(np.int32)), _dev(np.zeros(n, np.int64))
    q, k, v = (torch.zeros((n, h, D), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    out = torch.zeros_like(q)
    ws = torch.empty(B.decode_workspace_bytes(n, wide * 16, B.attn_desc(q, gpu.codes, tab, 0.1, k, out, kv_scales=gpu.scales)) + 16, dtype=torch.uint8, device="cuda")
    call = lambda: B.decode(q, gpu.codes, tab, lens, wide * 16, out, D ** -0.5, k_new=k, v_new=v, slot_mapping=slots, workspace=ws, kv_scales=gpu.scales)
    slots.fill_(-1)
    call()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            call()
    for step in range(1, 20):
        now = start + step
        x = [_rows(rng, n, h, D, "bf16") * np.float32(2.0 ** rng.integers(-3, 4)) for h in (hq, hkv, hkv)]
        sl = np.array([slot_of(s, now[s] - 1) for s in range(n)], np.int64)
        for t, a in zip((q, k, v), x):
            t.copy_(_dev(P.bf16(a), "bf16"))
        lens.copy_(_dev(now.astype(np.int32)))
        slots.copy_(_dev(sl))
        graphs[step % 2].replay()
        cache.append(P.bf16(x[1]), P.bf16(x[2]), sl)
        gpu.same(cache)
        _check(out, _want(cache, table, [(1, int(c)) for c in now], P.bf16(x[0])), "bf16", D, int(now.max()))


def test_rows_behind_the_last_sequence_stay(B):
    import torch
    rng = np.random.Generator(np.random.PCG64(12))
    lens = [(5, 20), (3, 3)]
    cache, table, slots, k, v = _batch(rng, lens, 1, 128, "bf16")
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    q = np.concatenate([_rows(rng, 8, 4, 128, "bf16"), np.zeros((4, 4, 128), np.float32)])
    kv = np.concatenate([np.stack([k, v]), np.zeros((2, 4, 1, 128), np.float32)], 1)
    out = torch.full((12, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    B.prefill(_dev(q, "bf16")[:8], gpu.codes, _dev(table), _dev(np.array([0, 5, 8], np.int32)), _dev(np.array([20, 3], np.int32)), 5, 20, out[:8], 128 ** -0.5,
              k_new=_dev(kv[0], "bf16"), v_new=_dev(kv[1], "bf16"), slot_mapping=_dev(np.r_[slots, [-1] * 4]), kv_scales=gpu.scales)
    gpu.same(cache)
    assert bool((out[8:] == 7).all())
    _check(out[:8], _want(cache, table, lens, q[:8]), "bf16", 128, 20)


def test_blocks_whose_offsets_pass_32_bits(B):
    """A cache of more than 2^32 bytes: append, prefill and decode of a sequence in its last blocks."""
    import torch
    rng = np.random.Generator(np.random.PCG64(13))
    D, far = 128, (1 << 20) + 9          # blocks of 4 KiB: 4 GiB and a little
    lens = [(20, 45)]
    cache, table, slots, k, v = _batch(rng, lens, 1, D, "bf16", num_blocks=9)
    codes = torch.zeros((far, 1, 2, 16 * D), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((far, 1, 2), dtype=torch.float32, device="cuda")
    codes[-9:], scales[-9:] = _dev(cache.codes), _dev(cache.scales)
    cache.append(k, v, slots)
    shift = far - 9
    q, out = _rows(rng, 20, 8, D, "bf16"), torch.empty((20, 8, D), dtype=torch.bfloat16, device="cuda")
    t, l = _dev(table + shift), _dev(np.array([45], np.int32))
    B.prefill(_dev(q, "bf16"), codes, t, _dev(np.array([0, 20], np.int32)), l, 20, 45, out, D ** -0.5, k_new=_dev(k, "bf16"), v_new=_dev(v, "bf16"),
              slot_mapping=_dev(slots + shift * 16), kv_scales=scales)
    assert np.array_equal(codes[-9:].cpu().numpy(), cache.codes) and np.array_equal(scales[-9:].cpu().numpy(), cache.scales)
    want = _want(cache, table, lens, q)
    _check(out, want, "bf16", D, 45)
    B.decode(_dev(q[-1:], "bf16"), codes, t, l, 45, out[:1], D ** -0.5, kv_scales=scales)
    _check(out[:1], [w[-1:] for w in want], "bf16", D, 45)


@pytest.mark.parametrize("dtype,D,hq,hkv", [("bf16", 128, 8, 1), ("f32", 64, 4, 1)])
def test_the_longest_max_seq_len(B, dtype, D, hq, hkv):
    """An upper bound of 2^31 - 1 tokens for contexts that are short."""
    import torch
    rng = np.random.Generator(np.random.PCG64(17))
    cache, table, slots, k, v = _batch(rng, [(3, 700)], hkv, D, dtype)
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    wide = torch.zeros((1, 2 ** 27), dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = _dev(table)
    q, longest = _rows(rng, 3, hq, D, dtype), 2 ** 31 - 1
    out, lens = torch.empty((3, hq, D), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda"), _dev(np.array([700], np.int32))
    B.prefill(_dev(q, dtype), gpu.codes, wide, _dev(np.array([0, 3], np.int32)), lens, 3, longest, out, D ** -0.5, k_new=_dev(k, dtype), v_new=_dev(v, dtype),
              slot_mapping=_dev(slots), kv_scales=gpu.scales)
    gpu.same(cache)
    want = _want(cache, table, [(3, 700)], q)
    _check(out, want, dtype, D, 700)
    B.decode(_dev(q[-1:], dtype), gpu.codes, wide, lens, longest, out[:1], D ** -0.5, kv_scales=gpu.scales)
    _check(out[:1], [w[-1:] for w in want], dtype, D, 700)


@pytest.mark.parametrize("option,value", [("OPT_GENERIC_ONLY", 1), ("OPT_PREFILL_TILE", 128), ("OPT_PREFILL_TILE", 256), ("OPT_PREFILL_SPLITS", 3)])
def test_kernels_chosen_by_option(B, option, value):
    """The general kernel on the shapes of the tuned ones, the wide prefill kernels, more key ranges."""
    import torch
    B.set_option(getattr(B, option), value)
    try:
        _prefill(B, "bf16", 128, 8, 1, [(70, 70), (133, 900), (1, 40)])
        if option == "OPT_GENERIC_ONLY":
            test_decode(B, "bf16", 128, 10, 2, [700, 0, 2, 31, 0, 95], True)
            test_mixed(B, "bf16", 128, 8, 1, [(70, 70), (33, 200)], [1, 17, 250, 64, 0])
    finally:
        B.set_option(getattr(B, option), 0)


def test_chunks_and_rows_in_one_launch(B):
    """A unified batch for which the plan puts the decode rows into the prefill kernel's launch, and the same batch with a workspace that
    only holds the two launches."""
    import torch
    rng = np.random.Generator(np.random.PCG64(15))
    D, hq, hkv = 128, 8, 1
    chunks, rows = [(300, 2300)], [int(c) for c in rng.integers(1, 2200, 60)]
    lens = chunks + [(1, c) for c in rows]
    cache, table, slots, k, v = _batch(rng, lens, hkv, D, "bf16")
    gpu = OnGpu(cache)
    cache.append(k, v, slots)
    q = _rows(rng, len(slots), hq, D, "bf16")
    want = _want(cache, table, lens, q)
    out = torch.empty((len(slots), hq, D), dtype=torch.bfloat16, device="cuda")
    dev = dict(q=_dev(q, "bf16"), t=_dev(table), cu=_dev(np.array([0, 300], np.int32)), l=_dev(np.array([c for _, c in lens], np.int32)))
    a = B.attn_desc(dev["q"], gpu.codes, dev["t"], D ** -0.5, None, out, kv_scales=gpu.scales)
    assert B.prefill_plan(1, 300, 300, 2300, a, 60, max(rows)).decode_wgs > 0
    both = B.mixed_workspace_bytes(1, 300, 300, 2300, 60, max(rows), a)
    least = max(B.prefill_workspace_bytes(1, 300, 300, 2300, a), B.decode_workspace_bytes(60, max(rows), a))
    new = dict(k_new=_dev(k, "bf16"), v_new=_dev(v, "bf16"), slot_mapping=_dev(slots))
    for i, size in enumerate((both, least)):
        ws = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
        B.mixed(dev["q"], gpu.codes, dev["t"], dev["cu"], dev["l"], 1, 300, 2300, max(rows), out, D ** -0.5, workspace=ws, kv_scales=gpu.scales,
                **(new if i == 0 else {}))
        gpu.same(cache)
        _check(out, want, "bf16", D, 2300)


def test_two_streams_at_once(B):
    """Batches of their own caches and workspaces on two streams, in flight together."""
    import torch
    rng = np.random.Generator(np.random.PCG64(16))
    lens, work = [(1, 60 + 31 * i) for i in range(50)], []
    for _ in range(2):
        cache, table, slots, k, v = _batch(rng, lens, 1, 128, "bf16")
        gpu = OnGpu(cache)
        cache.append(k, v, slots)
        q = _rows(rng, 50, 8, 128, "bf16")
        out = torch.empty((50, 8, 128), dtype=torch.bfloat16, device="cuda")
        args = (_dev(q, "bf16"), gpu.codes, _dev(table), _dev(np.array([c for _, c in lens], np.int32)), lens[-1][1], out, 128 ** -0.5)
        work.append((cache, gpu, args, dict(k_new=_dev(k, "bf16"), v_new=_dev(v, "bf16"), slot_mapping=_dev(slots), kv_scales=gpu.scales), _want(cache, table, lens, q)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(20):
        for st, (_, _, args, new, _) in zip(streams, work):
            with torch.cuda.stream(st):
                B.decode(*args, **new)
    torch.cuda.synchronize()
    for cache, gpu, args, _, want in work:
        gpu.same(cache)
        _check(args[5], want, "bf16", 128, lens[-1][1])
