"""Rotary positions against the formula in 64 bits, and what they have to leave alone.

How far a float32 result may be off: sine and cosine come from an angle in [-pi/4, pi/4] rounded to float32 (2^-24 of at most 0.79), a series
exact to 2e-9 and its five or so roundings, together below 2.5e-7; two products and a sum round by at most 2^-24 each of at most |a| + |b|.
That is below 5e-7 (|a| + |b|) |m|; bf16 rows are rounded once more, by at most 2^-8 of the result."""
import math

import numpy as np
import pytest

import plain_8bit as P
import plain_layer as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def _fused(rng, rows, heads, D, kind):
    import torch
    x = rng.standard_normal((rows, heads, D)).astype(np.float32)
    x = P.bf16(x) if kind == "bf16" else x
    return x, torch.from_numpy(x).to(DEV, torch.bfloat16 if kind == "bf16" else torch.float32)


def _np(t):
    return t.double().cpu().numpy()


def _close(got, before, turned, pos, f, kind, pairs, m):
    want = L.rotary(before[:, :turned], pos, f, pairs, m)
    there = (np.asarray(pos) >= 0)[:, None, None]
    rot = 2 * len(f)
    size = np.abs(before[:, :turned, :rot].astype(np.float64))
    other = np.flip(size.reshape(*size.shape[:2], -1, 2), -1).reshape(size.shape) if pairs else np.roll(size, rot // 2, -1)
    bound = 5e-7 * abs(m) * (size + other) + (2.0 ** -8 if kind == "bf16" else 2.0 ** -24) * np.abs(want[..., :rot]) + 1e-38
    assert (np.abs(got[:, :turned, :rot] - want[..., :rot]) <= np.where(there, bound, 0)).all()
    assert (got[:, :, rot:] == before[:, :, rot:]).all() and (got[:, turned:] == before[:, turned:]).all()      # the rest of the head, V


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rows,hq,hkv,D,rot", [(1, 8, 1, 128, 128), (97, 8, 1, 128, 128), (33, 5, 1, 128, 64), (7, 16, 2, 64, 64), (300, 4, 4, 64, 16), (3, 1, 1, 256, 256),
                                               (65, 10, 2, 72, 48), (9, 3, 1, 16, 16), (5000, 16, 2, 128, 96)])
def test_rows_by_their_positions(B, rows, hq, hkv, D, rot, pairs, kind):
    rng = np.random.Generator(np.random.PCG64(rows * 1000 + D + rot))
    x, buf = _fused(rng, rows, hq + 2 * hkv, D, kind)
    pos = rng.integers(0, 131072, rows)
    pos[0] = 0
    if rows > 4:
        pos[3], pos[rows // 2] = -1, -7                     # padding
    f, m = B.rotary_frequencies(rot, 500000.0)
    B.rotary(buf[:, :hq], buf[:, hq:hq + hkv], _i32(pos), f.to(DEV), pairs=pairs)
    _close(_np(buf), x, hq + hkv, pos, f.numpy(), kind, pairs, m)


def test_positions_up_to_the_end_of_int32(B):
    """The angle at 2^31 - 1: products in 64 bits, here against integers.  A frequency of 2 pi k / 2^40 turns 2^31 - 1 times k / 2^40."""
    import torch
    pos = np.array([2**31 - 1, 2**31 - 2, 2**30 + 1, 2**24 + 1, 123456789], np.int64)
    k = np.array([2**37, 3 * 2**35, 2**36, 5, 2**39 - 1, 2**40 - 3, 1, 2**20 + 1], np.int64)
    turns = np.array([[float(int(p) * int(q) % 2**40) / 2**40 for q in k] for p in pos])
    x = np.zeros((5, 1, 16), np.float32)
    x[..., :8] = 1
    q = torch.from_numpy(x).to(DEV)
    B.rotary(q, None, _i32(pos), torch.from_numpy(2 * math.pi * k / 2**40).to(DEV))
    got = _np(q)[:, 0]
    # 2 pi k / 2^40 in float64 and its quotient are off by 2^-52 of up to 2^31 turns: 2^-21 turns, 3e-6 radians
    assert np.abs(got[:, :8] - np.cos(2 * math.pi * turns)).max() < 3.1e-6 and np.abs(got[:, 8:] - np.sin(2 * math.pi * turns)).max() < 3.1e-6


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "wavelengths", "parts"])
def test_one_of_the_two_and_scalings(B, which, scaling):
    rng = np.random.Generator(np.random.PCG64(3))
    x, buf = _fused(rng, 41, 6, 128, "f32")
    f, m = B.rotary_frequencies(128, 10000.0, scaling, 8.0, 4096, 1.0, 32.0)
    pos = rng.integers(0, 32768, 41)
    heads = buf[:, :2]
    B.rotary(heads if which == "q" else None, heads if which == "k" else None, _i32(pos), f.to(DEV), magnitude=m)
    _close(_np(buf), x, 2, pos, f.numpy(), "f32", False, m)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("chunks,cached,decs,spare", [([5], [0], [], 0), ([3, 0, 40, 1], [7, 9, 0, 1000], [1, 0, 88, 131072, -3], 6), ([], [], [17, 4], 0), ([], [], [5], 9),
                                                      ([700, 1, 2], [0, 5, 6], [3], 0), ([0, 0], [4, 4], [9], 2)])
def test_rows_of_a_unified_batch(B, chunks, cached, decs, spare, kind):
    """Positions out of the lengths; rows set aside for chunks that were refused, and decode rows without a token, stay as they are."""
    rng = np.random.Generator(np.random.PCG64(sum(chunks) + len(decs)))
    cu = np.concatenate([[0], np.cumsum(chunks)]).astype(np.int64)
    total = int(cu[-1]) + spare
    pos = np.full(total + len(decs), -1, np.int64)
    for s, (n, c) in enumerate(zip(chunks, cached)):
        pos[cu[s]:cu[s] + n] = c + np.arange(n)
    pos[total:] = [max(d, 0) - 1 for d in decs]
    x, buf = _fused(rng, total + len(decs), 11, 64, kind)
    f, m = B.rotary_frequencies(64)
    B.rotary_mixed(buf[:, :8], buf[:, 8:9], _i32(cu), _i32([n + c for n, c in zip(chunks, cached)] + list(decs)), len(chunks), f.to(DEV), pairs=True)
    _close(_np(buf), x, 9, pos, f.numpy(), kind, True, m)


def test_turning_back(B):
    """Positions of the opposite angle undo a rotation, and a rotation keeps every pair's length."""
    import torch
    rng = np.random.Generator(np.random.PCG64(4))
    x, q = _fused(rng, 64, 4, 128, "f32")
    f, _ = B.rotary_frequencies(128)
    pos = _i32(rng.integers(0, 100000, 64))
    B.rotary(q, None, pos, f.to(DEV))
    size = lambda a: np.hypot(a[..., :64], a[..., 64:])
    assert np.abs(size(_np(q)) - size(x.astype(np.float64))).max() < 1e-5
    B.rotary(q, None, pos, -f.to(DEV))
    torch.cuda.synchronize()
    # two rotations, each off by 5e-7 (|a| + |b|) with |a| + |b| <= sqrt 2 times the pair's length
    assert (np.abs(_np(q) - x) <= 2 * 5e-7 * 2 * np.tile(size(x.astype(np.float64)), 2)).all()
