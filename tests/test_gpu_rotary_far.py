"""Rotary positions far out against whole-number arithmetic: t = position * frequency for the float64 value that the frequency is, its turns from
1 / (2 pi) to 60 places.  Sine and cosine may be off by 2.5e-7 (test_gpu_rotary says why), at whatever position."""
from fractions import Fraction
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("which", ["base 500000", "base 10000", "any"])
def test_angles_of_far_positions(B, which, pairs):
    import torch
    rng = np.random.Generator(np.random.PCG64(3))
    half = 64
    f = np.exp(rng.uniform(math.log(1e-7), math.log(1e3), half)) if which == "any" else B.rotary_frequencies(2 * half, float(which.split()[1]))[0].numpy()
    f[-1] = -f[-1]
    pos = np.concatenate([[2**31 - 1, 2**31 - 2, 2**31 - 12345, 2**30, 2**28 + 1, 2**27 - 1, 10**6 + 3, 131071, 1], rng.integers(2**28, 2**31, 60)])
    x = np.zeros((len(pos), 1, 2 * half), np.float32)
    x[..., slice(0, None, 2) if pairs else slice(0, half)] = 1
    q = torch.from_numpy(x).to(DEV)
    B.rotary(q, None, torch.from_numpy(pos.astype(np.int32)).to(DEV), torch.from_numpy(f).to(DEV), pairs=pairs)
    got = q.double().cpu().numpy()[:, 0]
    cos, sin = (got[:, 0::2], got[:, 1::2]) if pairs else (got[:, :half], got[:, half:])
    turns = [[float(int(p) * Fraction(float(v)) / (2 * PI) % 1) for v in f] for p in pos]
    t = 2 * math.pi * np.array(turns)
    assert np.abs(cos - np.cos(t)).max() <= 2.5e-7 and np.abs(sin - np.sin(t)).max() <= 2.5e-7
