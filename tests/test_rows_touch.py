"""Rows that share memory, found on the host whatever their strides (no GPU): the function against every pair of rows, and the calls that ask it."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

from paper_2509_16495_amd import build as BLD
from test_layer_refusals import B, PTR, _both, _norm


@pytest.fixture(scope="module")
def touch(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++ to compile the function for the host")
    d = str(tmp_path_factory.mktemp("touch"))
    src, lib = os.path.join(d, "touch.cpp"), os.path.join(d, "touch.so")
    with open(src, "w") as f:
        f.write('#include "rows_touch.h"\nextern "C" int touch(uint64_t a, int64_t la, int64_t sa, uint64_t b, int64_t lb, int64_t sb, int64_t n) '
                "{ return shiftattn::rows_touch(a, la, sa, b, lb, sb, n); }\n")
    subprocess.check_call(["g++", "-std=c++20", "-O1", "-shared", "-fPIC", "-I", BLD.CSRC, src, "-o", lib])
    f = ctypes.CDLL(lib).touch
    f.argtypes = [ctypes.c_uint64, ctypes.c_int64, ctypes.c_int64] * 2 + [ctypes.c_int64]
    return lambda *a: bool(f(*a))


def test_against_every_pair_of_rows(touch):
    rng, seen = random.Random(7), [0, 0]
    for _ in range(60000):
        n = rng.randint(1, 9)
        la, lb = rng.randint(1, 6), rng.randint(1, 6)
        sa, sb = la + rng.choice([0, rng.randint(0, 12), rng.randint(0, 60)]), lb + rng.choice([0, rng.randint(0, 12), rng.randint(0, 60)])
        if rng.random() < 0.2:
            sb = max(lb, sa * rng.choice([1, 2, 3]))
        a, b = rng.randint(100, 200), rng.randint(0, 700)
        want = any(a + i * sa < b + j * sb + lb and b + j * sb < a + i * sa + la for i in range(n) for j in range(n))
        assert touch(a, la, sa, b, lb, sb, n) == want, (a, la, sa, b, lb, sb, n)
        seen[want] += 1
    assert min(seen) > 5000


def test_rows_without_end(touch):
    """2^31 - 1 rows, places up to 2^62: distances that share a factor leave room, others meet somewhere."""
    n = 2**31 - 1
    assert not touch(2**40, 128, 4096, 2**40 + 128, 64, 8192, n) and touch(2**40, 128, 4096, 2**40 + 100, 64, 8192, n)
    assert touch(2**40, 128, 4096, 2**40 + 2048, 64, 8192 + 16, n)                  # 16 nearer each time
    assert not touch(2**40, 128, 2**30, 2**40 + n * 2**30, 64, 2**31, n) and touch(2**40, 128, 2**30, 2**40 + (n - 1) * 2**30 + 127, 64, 2**31, n)


def test_calls_whose_rows_are_at_different_distances(B):
    """bf16 rows are 128 bytes here, their codes 64, a float32 residual's 256."""
    codes = dict(out_format=B.CODES_INT8, scales=PTR + 0x9002, res=None, w=PTR + 0x8000)      # (a place of scales that is refused afterwards)
    refused = lambda **kw: _norm(B, **kw) == B.EINVAL and "share memory" in B.last_error()
    for at in (16, 64, 128, 448, 504, -8, -248):
        assert refused(**codes, out=PTR + at), at
    for at in (512, 4096, -256):
        assert _norm(B, **codes, out=PTR + at) == B.EINVAL and "share memory" not in B.last_error(), at
    f32 = dict(residual_dtype=B.F32, w=PTR + 0x8000, out=PTR + 0x4000, scales=PTR)            # scales beside values: refused afterwards
    for at in (16, 256, 496, -16, -1008):
        assert refused(**f32, res=PTR + at), at
    for at in (512, -1024):
        assert _norm(B, **f32, res=PTR + at) == B.EINVAL and "share memory" not in B.last_error(), at
    # codes in every other gap between rows, and half a row further
    assert not refused(**codes, out=PTR + 128, x_stride=256, out_stride=1024) and refused(**codes, out=PTR + 96, x_stride=256, out_stride=1024)
    # the residual's rows against out's
    assert refused(x=PTR + 0x4000, res=PTR, residual_dtype=B.F32, out=PTR + 1000 - 8, out_format=B.CODES_FP8, scales=PTR + 0x9002, w=PTR + 0x8000)
    # heads of q and k in one allocation, at different distances (2048 bytes a row of q)
    for k in (2048, 4096 + 512, 8192 - 256, 16):
        assert _both(B, k=PTR + k) == [B.EINVAL] * 2 and "heads" in B.last_error(), k
    assert _both(B, k=PTR + 8192, pos=PTR + 2, lens=PTR + 2) == [B.EINVAL] * 2 and "heads" not in B.last_error()
    assert _both(B, k=PTR + 2048, q_stride=2048, k_stride=4096, pos=PTR + 2, lens=PTR + 2) == [B.EINVAL] * 2 and "heads" not in B.last_error()
