"""Decode rows of heads of 64, many (row, head) pairs: the append launch in front of the attention takes every row for itself."""
import numpy as np
import pytest

import plain_8bit as P
from test_gpu_spare_rows import _dev, _rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,hkv", [(700, 6), (4100, 1)])
def test_decode_appends_many_rows(seqs, hkv):
    import torch
    from paper_2509_16495_amd import binding as B
    rng, D = np.random.Generator(np.random.PCG64(seqs)), 64
    lens = rng.integers(0, 18, seqs).astype(np.int32)          # padding rows, first tokens of a block, blocks that others fill
    table = rng.permutation(2 * seqs).astype(np.int32).reshape(seqs, 2)
    cache = P.Cache(2 * seqs, hkv, D)
    slot_of = lambda s, p: int(table[s, p // 16]) * 16 + p % 16
    for s, n in enumerate(lens):
        if n > 1:
            x = _rows(rng, int(n) - 1, hkv, 2 * D, dtype="bf16")
            cache.append(x[..., :D], x[..., D:], np.array([slot_of(s, p) for p in range(n - 1)]))
    codes, scales = _dev(cache.codes), _dev(cache.scales)
    slots = np.array([slot_of(s, n - 1) if n else -1 for s, n in enumerate(lens)], np.int64)
    kv, q = _rows(rng, seqs, hkv, 2 * D, dtype="bf16") * np.float32(4), _rows(rng, seqs, hkv, D, dtype="bf16")
    cache.append(kv[..., :D], kv[..., D:], slots)
    out = torch.full((seqs, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    B.decode(_dev(q, "bf16"), codes, _dev(table), _dev(lens), 32, out, 0.125, k_new=_dev(kv[..., :D], "bf16"), v_new=_dev(kv[..., D:], "bf16"),
             slot_mapping=_dev(slots), kv_scales=scales)
    assert np.array_equal(codes.cpu().numpy(), cache.codes) and np.array_equal(scales.cpu().numpy(), cache.scales)
    got = out.float().cpu().numpy()
    assert not got[lens == 0].any()
    for s in np.flatnonzero(lens)[::7]:
        want = P.attend(q[s:s + 1], cache, table[s], int(lens[s]), 0.125)
        assert (np.abs(got[s:s + 1] - want[0]) <= P.bound("bf16", *want, D, 17)).all()
