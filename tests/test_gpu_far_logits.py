"""Attention where float32 ends: keys whose logits are minus infinity, and queries and keys whose products leave the range of float32 unless
the keys' scale is in them.

In the first tests element 0 of q is 3e38, that of some keys -4 and that of the others 0: the former's logits are minus infinity in float32
(beyond -1e38 in 64 bits: a weight of 0 there too), the latter's are those of the remaining elements, exactly.  So the result is the softmax over
the others, and its error is bounded as that of a batch without element 0."""
import numpy as np
import pytest

import plain_8bit as P
from test_gpu_spare_rows import Values, _dev, _option, _rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


KINDS = [("scaled", "f32", 64, 4, 1), ("scaled", "bf16", 64, 4, 2), ("scaled", "bf16", 256, 2, 1), ("scaled", "bf16", 128, 8, 1), ("same", "bf16", 128, 8, 1),
         ("same", "f32", 64, 4, 1), ("same", "bf16", 80, 4, 1), ("same", "f32", 80, 2, 2)]
# tokens, and which of them are far below: a chunk of 64 or a group of 32 at the front, one per wavefront, in the middle, all but the last
PLACES = {"first": (300, lambda t: t < 64), "front": (300, lambda t: t < 200), "middle": (500, lambda t: (t >= 128) & (t < 320)), "late": (150, lambda t: t < 149),
          "many": (3000, lambda t: t < 2900), "turns": (2000, lambda t: t // 64 % 2 == 0), "groups": (400, lambda t: t // 32 % 2 == 0)}


class Batch:
    """One sequence; every row sees at least one key that is not far below.  `rows` last tokens are queries."""

    def __init__(self, fmt, dtype, D, hq, hkv, length, far, rows):
        rng = np.random.Generator(np.random.PCG64(length + D))
        t, n_blocks = np.arange(length), -(-length // 16)
        self.far, self.length, self.D, self.dtype = far(t), length, D, dtype
        assert all(not self.far[:length - rows + i + 1].all() for i in range(rows))
        kv = _rows(rng, length, hkv, 2 * D, dtype=dtype)
        kv[:, :, 0] = np.where(self.far, -4.0, 0.0)[:, None]
        self.cache = P.Cache(n_blocks, hkv, D) if fmt == "scaled" else Values(n_blocks, hkv, D)
        self.table = rng.permutation(n_blocks).astype(np.int32)[None]
        slots = self.table[0, t // 16].astype(np.int64) * 16 + t % 16
        self.cache.append(kv[..., :D], kv[..., D:], slots)
        self.kw = dict(kv_scales=_dev(self.cache.scales)) if fmt == "scaled" else {}
        self.codes = _dev(self.cache.codes) if fmt == "scaled" else self.cache.device(dtype)
        self.q = _rows(rng, rows, hq, D, dtype=dtype)
        self.q[:, :, 0] = 0
        q = self.q.copy()
        q[:, :, 0] = P.bf16(np.float32(3e38))
        self.dev = dict(q=_dev(q, dtype), table=_dev(self.table), lens=_dev(np.array([length], np.int32)))

    def check(self, got):
        got, rows = got.float().cpu().numpy().astype(np.float64), len(self.q)
        hq, heads, D = self.q.shape[1], self.cache.heads, self.D
        hidden = (np.arange(self.length) > np.arange(self.length - rows, self.length)[:, None]) | self.far
        for j in range(hq):
            k, v = (self.cache.rows(self.table[0], self.length, j // (hq // heads), x) for x in (0, 1))
            q = self.q[:, j].astype(np.float64)
            s = np.where(hidden, -np.inf, q @ k.T * D ** -0.5)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            big = np.where(hidden, 0, np.abs(q) @ np.abs(k).T).max(1)[:, None] * D ** -0.5
            off = np.abs(got[:, j] - p @ v) / P.bound(self.dtype, p @ v, p @ np.abs(v), big, D, self.length)
            assert np.isfinite(got[:, j]).all() and off.max() <= 1.0, off.max()


def _out(b):
    import torch
    return torch.empty(b.q.shape, dtype=torch.bfloat16 if b.dtype == "bf16" else torch.float32, device="cuda")


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("fmt,dtype,D,hq,hkv", KINDS)
@pytest.mark.parametrize("place", PLACES)
def test_decode_over_keys_far_below(B, fmt, dtype, D, hq, hkv, place, generic):
    b = Batch(fmt, dtype, D, hq, hkv, *PLACES[place], 1)
    out = _out(b)
    with _option(B, "OPT_GENERIC_ONLY" if generic else None, 1):
        B.decode(b.dev["q"], b.codes, b.dev["table"], b.dev["lens"], b.length, out, D ** -0.5, **b.kw)
    b.check(out)


@pytest.mark.parametrize("generic", [False, True])
@pytest.mark.parametrize("fmt,dtype,D,hq,hkv", KINDS)
@pytest.mark.parametrize("place", [p for p in PLACES if p != "late"])
def test_prefill_over_keys_far_below(B, fmt, dtype, D, hq, hkv, place, generic):
    b = Batch(fmt, dtype, D, hq, hkv, *PLACES[place], 40)
    out = _out(b)
    with _option(B, "OPT_GENERIC_ONLY" if generic else None, 1):
        B.prefill(b.dev["q"], b.codes, b.dev["table"], _dev(np.array([0, 40], np.int32)), b.dev["lens"], 40, b.length, out, D ** -0.5, **b.kw)
    b.check(out)


@pytest.mark.parametrize("fmt", ["scaled", "same"])
def test_decode_rows_beside_chunks_over_keys_far_below(B, fmt):
    """Decode rows in the prefill kernel's launch, which take another reference: 60 of one sequence's blocks each."""
    import torch
    b = Batch(fmt, "bf16", 128, 8, 1, 2000, lambda t: t // 32 % 3 > 0, 1)
    table, lens = b.dev["table"].repeat(61, 1), b.dev["lens"].repeat(61)
    q = torch.cat([torch.zeros((300, 8, 128), dtype=torch.bfloat16, device="cuda"), b.dev["q"].repeat(60, 1, 1)])
    out = torch.empty_like(q)
    assert B.prefill_plan(1, 300, 300, 2000, B.attn_desc(q, b.codes, table, 128 ** -0.5, None, out, **b.kw), 60, 2000).decode_wgs > 0
    B.mixed(q, b.codes, table, _dev(np.array([0, 300], np.int32)), lens, 1, 300, 2000, 2000, out, 128 ** -0.5, **b.kw)
    for i in (0, 31, 59):
        b.check(out[300 + i:301 + i])


@pytest.mark.parametrize("dtype,D", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 256)])
@pytest.mark.parametrize("q_size,k_size", [(2.0 ** 122, 2.0 ** -95), (2.0 ** -123, 2.0 ** 116)])
def test_products_are_of_what_the_cache_stands_for(B, dtype, D, q_size, k_size):
    """q times a code would pass 2^128 where the block's scale is small, and lie at the bottom of the range where it is large; q times the
    key's value stays near 1."""
    import torch
    rng = np.random.Generator(np.random.PCG64(D))
    length, rows, scale = 200, 5, 1.0 / (q_size * k_size) / D ** 0.5
    t = np.arange(length)
    cache = P.Cache(13, 1, D)
    kv = _rows(rng, length, 1, 2 * D, dtype=dtype)
    kv[..., :D] *= np.float32(k_size)
    table = rng.permutation(13).astype(np.int32)[None]
    cache.append(kv[..., :D], kv[..., D:], table[0, t // 16].astype(np.int64) * 16 + t % 16)
    q = _rows(rng, rows, 4, D, dtype=dtype) * np.float32(q_size)
    out = torch.empty((rows, 4, D), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    codes, scales = _dev(cache.codes), _dev(cache.scales)
    for call in ("prefill", "decode"):
        if call == "prefill":
            B.prefill(_dev(q, dtype), codes, _dev(table), _dev(np.array([0, rows], np.int32)), _dev(np.array([length], np.int32)), rows, length, out, scale, kv_scales=scales)
            got, want = out, P.attend(q, cache, table[0], length, scale)
        else:
            B.decode(_dev(q[-1:], dtype), codes, _dev(table), _dev(np.array([length], np.int32)), length, out[:1], scale, kv_scales=scales)
            got, want = out[:1], P.attend(q[-1:], cache, table[0], length, scale)
        got = got.float().cpu().numpy().astype(np.float64)
        off = np.abs(got - want[0]) / P.bound(dtype, *want, D, length)
        assert np.isfinite(got).all() and off.max() <= 1.0, (call, off.max())
