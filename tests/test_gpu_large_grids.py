"""Calls whose work would be more threads than one launch can have (2^32 - 1; a larger one drops the rest without a word): nothing is left
out.  Few of the rows have much work, so that the calls are quick."""
import numpy as np
import pytest

import plain_8bit as P
from test_gpu_spare_rows import Values, _dev, _rows

pytestmark = pytest.mark.gpu

D, SCALE = 16, 0.25


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _cache(rng, lengths, heads):
    """A cache of these sequences, and their table (sequence by sequence, blocks in order)."""
    wide = max(-(-n // 16) for n in lengths)
    cache, table = P.Cache(wide * len(lengths), heads, D), np.arange(wide * len(lengths), dtype=np.int32).reshape(len(lengths), wide)
    for s, n in enumerate(lengths):
        x = _rows(rng, n, heads, 2 * D, dtype="bf16")
        cache.append(x[..., :D], x[..., D:], table[s, np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16)
    return cache, table


def _close(got, want, keys):
    off = np.abs(got.float().cpu().numpy() - want[0]) / P.bound("bf16", *want, D, keys)
    assert off.max() <= 1.0


def test_decode_of_many_padding_rows(B):
    import torch
    rng, rows, at = np.random.Generator(np.random.PCG64(1)), (1 << 24) + 37, [0, 1000, (1 << 24) - 1, 1 << 24, (1 << 24) + 36]
    lengths = [300, 17, 40, 1024, 5]
    cache, small = _cache(rng, lengths, 1)
    table = torch.zeros((rows, small.shape[1]), dtype=torch.int32, device="cuda")
    table[at] = _dev(small)
    lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    lens[at] = _dev(np.array(lengths, np.int32))
    q, qs = torch.zeros((rows, 1, D), dtype=torch.bfloat16, device="cuda"), _rows(rng, 5, 1, D, dtype="bf16")
    q[at] = _dev(qs, "bf16")
    out = torch.full_like(q, 7.0)
    B.decode(q, _dev(cache.codes), table, lens, 1024, out, SCALE, kv_scales=_dev(cache.scales))
    for i, (row, n) in enumerate(zip(at, lengths)):
        _close(out[row:row + 1], P.attend(qs[i:i + 1], cache, small[i], n, SCALE), n)
    out[at] = 0
    assert not bool(out.any())


def test_prefill_of_many_chunks(B):
    """Chunks of one token, most of them alone in the first block: their result is its V."""
    import torch
    rng, rows, at = np.random.Generator(np.random.PCG64(2)), (1 << 24) + 37, [5, (1 << 24) - 1, (1 << 24) + 1]
    lengths = [300, 40, 33]
    cache, small = _cache(rng, lengths, 1)
    table, lens = torch.zeros((rows, small.shape[1]), dtype=torch.int32, device="cuda"), torch.ones(rows, dtype=torch.int32, device="cuda")
    table[at], lens[at] = _dev(small), _dev(np.array(lengths, np.int32))
    qs = _rows(rng, 3, 1, D, dtype="bf16")
    q = torch.ones((rows, 1, D), dtype=torch.bfloat16, device="cuda")
    q[at] = _dev(qs, "bf16")
    out = torch.full_like(q, 7.0)
    B.prefill(q, _dev(cache.codes), table, torch.arange(rows + 1, dtype=torch.int32, device="cuda"), lens, 1, 300, out, SCALE, kv_scales=_dev(cache.scales))
    for i, (row, n) in enumerate(zip(at, lengths)):
        _close(out[row:row + 1], P.attend(qs[i:i + 1], cache, small[i], n, SCALE), n)
    first = _dev(cache.rows(small[0], 1, 0, 1).astype(np.float32), "bf16")   # (E4M3 times a power of two: a bf16 value)
    out[at] = first
    assert bool((out == first).all())


def test_append_of_many_padding_rows(B):
    import torch
    rng, heads, tokens = np.random.Generator(np.random.PCG64(3)), 64, (1 << 20) + 40
    cache = P.Cache(4, heads, D, rng)
    codes, scales = _dev(cache.codes), _dev(cache.scales)
    slots, kv = np.full(tokens, -1, np.int64), np.zeros((20, heads, 2 * D), np.float32)
    kv[:] = _rows(rng, 20, heads, 2 * D, dtype="bf16")
    at = np.r_[0:3, (1 << 20) - 3:(1 << 20) + 4, tokens - 10:tokens]   # runs at both ends and across the line
    slots[at] = np.r_[5:8, 16:23, 38:48]
    rows = torch.zeros((tokens, heads, 2 * D), dtype=torch.bfloat16, device="cuda")
    rows[at] = _dev(kv, "bf16")
    cache.append(kv[..., :D], kv[..., D:], slots[at])
    B.kv_write(rows[..., :D].contiguous(), rows[..., D:].contiguous(), _dev(slots), codes, kv_scales=scales)
    got, nan = codes.cpu().numpy(), (cache.codes & 0x7F) == 0x7F      # (what the blocks' first tokens hold is random: a NaN code may change its sign)
    assert np.array_equal(scales.cpu().numpy(), cache.scales)
    assert np.array_equal(got[~nan], cache.codes[~nan]) and np.all((got[nan] & 0x7F) == 0x7F)


def test_quantiser_of_many_rows(B):
    import torch
    rng, rows = np.random.Generator(np.random.PCG64(4)), (1 << 24) + 37
    part = P.bf16(rng.standard_normal((1 << 12, 8)).astype(np.float32))
    x = _dev(part, "bf16").repeat(rows // len(part) + 1, 1)[:rows].contiguous()
    codes, scales = torch.full((rows, 8), 99, dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
    B.quantize_rows_int8(x, codes, scales)
    want, scale = (_dev(a) for a in P.quantise_int8(part))
    whole = rows // len(part) * len(part)
    for got, part in ((codes, want), (scales, scale)):
        assert bool((got[:whole].view(-1, *part.shape) == part).all()) and torch.equal(got[whole:], part[:rows - whole])


def test_general_kernel_on_many_padding_rows(B):
    """A cache without scales, four heads a row."""
    import torch
    rng, rows, at = np.random.Generator(np.random.PCG64(5)), (1 << 24) + 37, [3, (1 << 24) - 2, (1 << 24) + 2]
    lengths = [70, 40, 33]
    cache, small = Values(15, 1, D), np.arange(15, dtype=np.int32).reshape(3, 5)
    for s, n in enumerate(lengths):
        x = _rows(rng, n, 1, 2 * D, dtype="bf16")
        cache.append(x[..., :D], x[..., D:], small[s, np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16)
    table, lens = torch.zeros((rows, 5), dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    table[at], lens[at] = _dev(small), _dev(np.array(lengths, np.int32))
    qs = _rows(rng, 3, 4, D, dtype="bf16")
    q = torch.zeros((rows, 4, D), dtype=torch.bfloat16, device="cuda")
    q[at] = _dev(qs, "bf16")
    out = torch.full_like(q, 7.0)
    B.decode(q, cache.device("bf16"), table, lens, 70, out, SCALE)
    for i, (row, n) in enumerate(zip(at, lengths)):
        _close(out[row:row + 1], P.attend(qs[i:i + 1], cache, small[i], n, SCALE), n)
    out[at] = 0
    assert not bool(out.any())
