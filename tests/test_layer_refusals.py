"""What the operators around the projections and decode_shared refuse, the C ABI by code and the Python calls by exception, before anything
is enqueued; and the frequencies of rotary positions (no GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

BF, F32, F64, U8, I8, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.int8, torch.int32, torch.int64
PTR = 0x10000   # aligned, and never followed: every call below is refused on the host


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    if not binding.is_built():
        import __graft_entry__
        __graft_entry__.build()
    binding.lib()
    return binding


def _z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


def _accepted():
    """Any call's arguments are fine but for the place they are in: the last thing asked about."""
    return pytest.raises(RuntimeError, match="a tensor on the GPU is wanted")


# ---- add_rms_norm ------------------------------------------------------------------------------------------------------
def _norm(B, x=PTR, res=PTR, w=PTR + 128, out=PTR + 64, scales=None, rows=4, **kw):
    n = B.Norm(cols=64, x_dtype=B.BF16, residual_dtype=B.BF16, weight_dtype=B.BF16, out_format=B.BF16, eps=1e-5)
    for k, v in kw.items():
        setattr(n, k, v)
    return B.lib().shiftattn_add_rms_norm(x, res, w, out, scales, rows, ctypes.byref(n), None)


def test_norm_refuses(B):
    assert B.lib().shiftattn_add_rms_norm(PTR, PTR, PTR, PTR, None, 1, None, None) == B.EINVAL
    for kw in (dict(x_dtype=2), dict(weight_dtype=-1), dict(residual_dtype=7), dict(out_format=4), dict(out_format=-1), dict(reserved=1), dict(rows=-1), dict(cols=0),
               dict(cols=-8), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(weight_offset=math.nan), dict(weight_offset=math.inf),
               dict(x_stride=56), dict(residual_stride=56), dict(out_stride=56), dict(x_stride=68), dict(residual_stride=68), dict(out_stride=68), dict(x_stride=-64),
               dict(x=None), dict(w=None), dict(out=None), dict(x=PTR + 8), dict(res=PTR + 8), dict(w=PTR + 8), dict(out=PTR + 8), dict(scales=PTR),
               dict(out_format=B.CODES_INT8), dict(out_format=B.CODES_FP8, scales=PTR + 2), dict(out_format=B.CODES_FP8, scales=PTR, out=PTR + 4),
               dict(out_format=B.CODES_INT8, scales=PTR, out_stride=68),
               dict(out=PTR),                                                                          # the residual's rows
               dict(res=None, out=PTR, out_format=B.F32), dict(res=None, out=PTR, out_stride=128), dict(res=None, out=PTR, out_format=B.CODES_FP8, scales=PTR),
               dict(residual_dtype=B.F32), dict(residual_stride=128)):                                 # x in another type or with another stride
        assert _norm(B, **kw) == B.EINVAL, kw
        assert B.last_error()
    for cols in (4, 63, 65544, 1 << 30):
        assert _norm(B, cols=cols) == B.EUNSUPPORTED
    assert _norm(B, rows=0) == B.OK and _norm(B, rows=0, x=None, w=None, out=None) == B.OK
    assert _norm(B, rows=0, residual_dtype=9) == B.EINVAL and _norm(B, rows=0, residual_dtype=9, res=None) == B.OK   # not read without a residual


def test_norm_python_refuses(B):
    ok = dict(x=_z(5, 64), w=_z(64), out=_z(5, 64), res=_z(5, 64), scales=None, eps=1e-5)
    call = lambda **kw: (lambda a: B.add_rms_norm(a["x"], a["w"], a["out"], a["eps"], residual=a["res"], scales=a["scales"]))({**ok, **kw})
    wide = _z(5, 80)
    s = _z(5, dtype=F32)
    for kw in ({}, dict(res=None), dict(x=wide[:, :64]), dict(res=_z(5, 64, dtype=F32)), dict(out=_z(5, 64, dtype=F32)), dict(out=_z(5, 64, dtype=U8), scales=s),
               dict(out=_z(5, 64, dtype=I8), scales=s), dict(w=_z(64, dtype=F32))):
        with _accepted():
            call(**kw)
    for kw, error in [(dict(x=_z(5, 64, dtype=torch.float16)), TypeError), (dict(x=_z(320)), ValueError), (dict(out=_z(5, 56)), AssertionError), (dict(res=_z(4, 64)), AssertionError),
                      (dict(w=_z(56)), AssertionError), (dict(w=_z(128)[::2]), AssertionError), (dict(w=_z(1, 64)), AssertionError), (dict(out=_z(5, 64, dtype=U8)), AssertionError),
                      (dict(scales=s), AssertionError), (dict(out=_z(5, 64, dtype=I8), scales=_z(4, dtype=F32)), AssertionError), (dict(out=_z(5, 64, dtype=I8), scales=_z(5)), AssertionError),
                      (dict(x=_z(64, 5).t()), AssertionError), (dict(res=_z(1, 64).expand(5, 64)), AssertionError), (dict(out=_z(1, 64).expand(5, 64)), AssertionError),
                      (dict(x=None), TypeError), (dict(eps="x"), TypeError), (dict(out=_z(5, 64, dtype=I32)), TypeError)]:
        with pytest.raises(error):
            call(**kw)
            pytest.fail(str(kw))


# ---- rotary ------------------------------------------------------------------------------------------------------------
def _desc(B, **kw):
    r = B.Rotary(num_q_heads=8, num_kv_heads=1, head_dim=128, rot_dim=128, dtype=B.BF16, magnitude=1.0)
    for k, v in kw.items():
        setattr(r, k, v)
    return ctypes.byref(r)


def _both(B, q=PTR, k=PTR + 2048, f=PTR, rows=4, pos=PTR, cu=PTR, lens=PTR, chunks=1, **kw):
    L, r = B.lib(), _desc(B, **kw)
    return [L.shiftattn_rotary(q, k, pos, rows, f, r, None), L.shiftattn_rotary_mixed(q, k, cu, lens, chunks, rows, 0, f, r, None)]


def test_struct_layouts_match_header(B):
    assert ctypes.sizeof(B.Norm) == 8 * 4 + 3 * 8 and B.Norm.x_stride.offset == 32 and B.Norm.eps.offset == 20
    assert ctypes.sizeof(B.Rotary) == 8 * 4 + 2 * 8 and B.Rotary.magnitude.offset == 24 and B.Rotary.q_stride.offset == 32


def test_rotary_refuses(B):
    L = B.lib()
    assert L.shiftattn_rotary(PTR, PTR, PTR, 1, PTR, None, None) == B.EINVAL and L.shiftattn_rotary_mixed(PTR, PTR, PTR, PTR, 1, 1, 1, PTR, None, None) == B.EINVAL
    for kw in (dict(dtype=2), dict(layout=2), dict(layout=-1), dict(reserved=1), dict(num_q_heads=0), dict(num_kv_heads=-1), dict(num_q_heads=65537), dict(head_dim=0),
               dict(rot_dim=0), dict(rot_dim=144), dict(magnitude=math.nan), dict(magnitude=-math.inf), dict(q_stride=1016), dict(k_stride=120), dict(q_stride=1028),
               dict(k_stride=132), dict(rows=-1), dict(f=None), dict(f=PTR + 4), dict(q=None, k=None), dict(q=PTR + 8), dict(k=PTR + 8), dict(k=PTR)):
        assert _both(B, **kw) == [B.EINVAL] * 2, kw
    for kw in (dict(rot_dim=24), dict(rot_dim=8), dict(head_dim=132), dict(head_dim=264, rot_dim=256), dict(rot_dim=2)):
        assert _both(B, **kw) == [B.EUNSUPPORTED] * 2, kw
    assert _both(B, pos=None, cu=None) == [B.EINVAL] * 2 and _both(B, pos=PTR + 2, lens=None) == [B.EINVAL] * 2 and _both(B, pos=None, lens=PTR + 2) == [B.EINVAL] * 2
    r = _desc(B)
    for counts in ((-1, 1, 1), (1, -1, 1), (1, 1, -1)):
        assert L.shiftattn_rotary_mixed(PTR, PTR, PTR, PTR, *counts, PTR, r, None) == B.EINVAL
    assert L.shiftattn_rotary_mixed(PTR, PTR, PTR, PTR, 1, 2**31 - 1, 1, PTR, r, None) == B.EUNSUPPORTED
    assert _both(B, rows=0, q=None, k=None, f=None, pos=None, cu=None, lens=None) == [B.OK] * 2


def test_rotary_python_refuses(B):
    ok = dict(q=_z(5, 8, 64), k=_z(5, 1, 64), pos=_z(5, dtype=I32), cu=_z(2, dtype=I32), lens=_z(3, dtype=I32), chunks=1, f=_z(32, dtype=F64), m=1.0)

    def calls(**kw):
        a = {**ok, **kw}
        return [lambda: B.rotary(a["q"], a["k"], a["pos"], a["f"], magnitude=a["m"]), lambda: B.rotary_mixed(a["q"], a["k"], a["cu"], a["lens"], a["chunks"], a["f"], magnitude=a["m"])]
    fused = _z(5, 10, 64)
    for kw in ({}, dict(q=None), dict(k=None), dict(q=fused[:, :8], k=fused[:, 8:9]), dict(f=_z(16, dtype=F64)), dict(q=_z(5, 8, 64, dtype=F32), k=None)):
        for call in calls(**kw):
            with _accepted():
                call()
    for kw, error in [(dict(q=None, k=None), AssertionError), (dict(q=_z(5, 512)), ValueError), (dict(k=_z(4, 1, 64)), AssertionError), (dict(k=_z(5, 1, 128)), AssertionError),
                      (dict(k=_z(5, 1, 64, dtype=F32)), AssertionError), (dict(f=_z(33, dtype=F64)), AssertionError), (dict(f=_z(32, dtype=F32)), AssertionError),
                      (dict(f=_z(64, dtype=F64)[::2]), AssertionError), (dict(q=_z(8, 5, 64).transpose(0, 1)), AssertionError), (dict(q=_z(1, 8, 64).expand(5, 8, 64)), AssertionError),
                      (dict(q=_z(5, 8, 64, dtype=torch.float16), k=None), TypeError), (dict(m="x"), TypeError)]:
        for call in calls(**kw):
            with pytest.raises(error):
                call()
                pytest.fail(str(kw))
    for kw in (dict(pos=_z(4, dtype=I32)), dict(pos=_z(5, dtype=I64)), dict(pos=_z(10, dtype=I32)[::2])):
        with pytest.raises(AssertionError):
            calls(**kw)[0]()
    for kw in (dict(cu=_z(3, dtype=I32)), dict(cu=_z(2, dtype=I64)), dict(lens=_z(3, dtype=I64)), dict(lens=_z(7, dtype=I32)), dict(chunks=-1), dict(chunks=4, cu=_z(5, dtype=I32)),
               dict(cu=_z(4, dtype=I32)[::2]), dict(lens=_z(6, dtype=I32)[::2])):
        with pytest.raises(AssertionError):
            calls(**kw)[1]()


def test_rows_that_share_memory(B):
    """Rows that cross, found on the host where their distance is the same; rows side by side, between each other and behind each other are not."""
    row = 64 * 2
    norm = lambda **kw: _norm(B, **{**dict(x=PTR, res=None, out=PTR + 8192, w=PTR + 0x8000), **kw})
    for at in (16, row - 16, row, 3 * row, 4 * row - 16, -16, -row, -4 * row + 16):
        assert norm(out=PTR + at) == B.EINVAL and "share memory" in B.last_error()
        assert norm(res=PTR + at) == B.EINVAL and norm(res=PTR + 8192 + at) == B.EINVAL
        assert norm(out=PTR + at, x_stride=32 + 64, out_stride=32 + 64) == B.EINVAL
    assert norm(out=PTR + 16, rows=1, out_stride=128) == B.EINVAL and norm(out=PTR + 16, out_format=B.F32, out_stride=64, x_stride=128) == B.EINVAL
    # heads 0 .. 7 and 8 of rows of ten are apart, heads 0 .. 7 and 7 are not, nor heads 9 .. 16 of rows of ten and 7 (the first of the next row)
    fused = dict(q_stride=1280, k_stride=1280)
    for k in (7, -9, 10 - 1 - 9, 37, 30):
        assert _both(B, k=PTR + 256 * k, **fused) == [B.EINVAL] * 2 and "heads" in B.last_error(), k
    assert _both(B, k=PTR + 1024, rows=1) == [B.EINVAL] * 2
    # side by side: refused for what comes behind in the order of the checks
    for k in (8, 9, -1, -2, 40, 38):
        assert _both(B, k=PTR + 256 * k, pos=PTR + 2, lens=PTR + 2, **fused) == [B.EINVAL] * 2 and "heads" not in B.last_error(), k
    assert _both(B, k=PTR + 2048, rows=1, pos=None, lens=None) == [B.EINVAL] * 2 and "heads" not in B.last_error()


def test_frequencies(B):
    """Each scaling from its definition, and at the ends where it changes nothing or divides by the factor."""
    i = np.arange(64)
    plain = 10000.0 ** (-2.0 * i / 128)
    get = lambda *a: (lambda f, m: (f.numpy(), m))(*B.rotary_frequencies(128, 10000.0, *a))
    f, m = get()
    assert np.allclose(f, plain, rtol=1e-15) and m == 1.0
    f, m = get("linear", 4.0)
    assert np.allclose(f, plain / 4, rtol=1e-15) and m == 1.0
    f, m = get("base", 4.0)
    assert f[0] == 1.0 and np.isclose(f[63], plain[63] / 4, rtol=1e-13) and (f[1:63] < plain[1:63]).all() and (f[1:63] > plain[1:63] / 4).all()
    L, turns = 8192.0, 8192.0 * plain / (2 * np.pi)
    f, m = get("wavelengths", 8.0, L, 1.0, 4.0)
    assert np.allclose(f[turns >= 4], plain[turns >= 4], rtol=1e-15) and np.allclose(f[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15) and m == 1.0
    s = (turns - 1) / 3
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.allclose(f[mid], (s * plain + (1 - s) * plain / 8)[mid], rtol=1e-14)
    f, m = get("parts", 4.0, 4096.0, 1.0, 32.0)
    at = lambda x: 128 * math.log(4096 / (2 * math.pi * x)) / (2 * math.log(10000.0))
    lo, hi = math.floor(at(32.0)), math.ceil(at(1.0))
    assert 0 < lo < hi < 64
    s = 1 - np.clip((i - lo) / (hi - lo), 0, 1)
    assert np.allclose(f, s * plain + (1 - s) * plain / 4, rtol=1e-14) and m == np.float32(0.1 * math.log(4.0) + 1)
    assert get("parts", 1.0, 4096.0)[1] == 1.0 and np.allclose(get("parts", 1.0, 4096.0)[0], plain, rtol=1e-14)
    for kw in (dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=7), dict(rot_dim=2, scaling="base"), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(scaling="linear", factor=0.5),
               dict(scaling="linear", factor=math.nan), dict(scaling="parts", factor=2.0), dict(scaling="parts", factor=2.0, original_len=100.0, low=2.0, high=1.0),
               dict(scaling="wavelengths", factor=2.0, original_len=-5.0), dict(scaling="wavelengths", factor=2.0, original_len=5.0, low=0.0), dict(scaling="base", base=1e300, factor=1e300)):
        with pytest.raises(B.ShiftAttnError) as e:
            B.rotary_frequencies(**{"rot_dim": 128, **kw})
        assert e.value.code == B.EINVAL
    with pytest.raises(ValueError):
        B.rotary_frequencies(128, scaling="other")
    out, mag = (ctypes.c_double * 8)(), ctypes.c_float()
    assert B.lib().shiftattn_rotary_frequencies(5, 16, 1e4, 1, 0, 0, 0, out, ctypes.byref(mag)) == B.EINVAL
    assert B.lib().shiftattn_rotary_frequencies(0, 16, 1e4, 1, 0, 0, 0, None, ctypes.byref(mag)) == B.EINVAL
    assert B.lib().shiftattn_rotary_frequencies(0, 16, 1e4, 1, 0, 0, 0, out, None) == B.EINVAL


# ---- decode_shared -----------------------------------------------------------------------------------------------------
def _attn(B, **kw):
    a = B.Attn(num_q_heads=8, num_kv_heads=1, head_dim=128, dtype=B.BF16, block_size=16, num_blocks=64, max_blocks_per_seq=8, softmax_scale=0.1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _shared(B, a, q=PTR, k=None, v=None, slots=None, cache=PTR, scales=None, table=PTR, lens=PTR, seqs=3, ms=64, off=PTR, sh=PTR, groups=1, out=PTR, ws=PTR, wsb=1 << 30):
    return B.lib().shiftattn_decode_shared(q, k, v, slots, cache, scales, table, lens, seqs, ms, off, sh, groups, out, ws, wsb, None if a is None else ctypes.byref(a), None)


def test_decode_shared_refuses(B):
    assert _shared(B, None) == B.EINVAL
    a = _attn(B)
    for kw in (dict(q=None), dict(cache=None), dict(table=None), dict(lens=None), dict(out=None), dict(off=None), dict(sh=None), dict(off=PTR + 2), dict(sh=PTR + 1), dict(groups=-1),
               dict(seqs=-1), dict(ms=-1), dict(ms=129), dict(k=PTR), dict(v=PTR, slots=PTR), dict(q=PTR + 8), dict(out=PTR + 8), dict(cache=PTR + 8), dict(scales=PTR),
               dict(k=PTR + 8, v=PTR, slots=PTR)):
        assert _shared(B, a, **kw) == B.EINVAL, kw
    for kw in (dict(num_kv_heads=3), dict(dtype=4), dict(softmax_scale=0.0), dict(q_stride=8), dict(reserved=2), dict(kv_format=B.KV_FP8_E4M3), dict(kv_format=9),
               dict(kv_format=B.KV_FP8_E4M3_BLOCKS)):
        assert _shared(B, _attn(B, **kw)) == B.EINVAL, kw
    assert _shared(B, _attn(B, kv_format=B.KV_FP8_E4M3_BLOCKS), scales=PTR + 4) == B.EINVAL
    assert _shared(B, _attn(B, block_size=32)) == B.EUNSUPPORTED and _shared(B, _attn(B, head_dim=100)) == B.EUNSUPPORTED
    need = B.decode_shared_workspace_bytes(3, 64, 1, a)
    assert 0 < need < 1 << 30
    for kw in (dict(ws=None), dict(wsb=need - 1), dict(ws=PTR + 8), dict(wsb=0)):
        assert _shared(B, a, **kw) == B.EWORKSPACE, kw
    assert _shared(B, a, seqs=0) == B.OK
    big = 2**64 - 1
    assert B.decode_shared_workspace_bytes(3, 64, -1, a) == big and B.decode_shared_workspace_bytes(-1, 64, 1, a) == big and B.decode_shared_workspace_bytes(3, -1, 1, a) == big
    assert B.decode_shared_workspace_bytes(3, 64, 1, _attn(B, head_dim=7)) == big
    assert B.decode_shared_workspace_bytes(0, 64, 0, a) == 0 == B.decode_shared_workspace_bytes(3, 64, 1, _attn(B, dtype=B.F32))


def test_the_option_and_the_sizes_that_follow_it(B):
    a = _attn(B, max_blocks_per_seq=4000)
    assert B.get_option(B.OPT_DECODE_SHARED) == 0
    for value in (-1, 3):
        assert B.lib().shiftattn_set_option(B.OPT_DECODE_SHARED, value) == B.EINVAL
    plain = lambda n, ms: B.decode_workspace_bytes(n, ms, a)
    shared = lambda n, ms, groups=2: B.decode_shared_workspace_bytes(n, ms, groups, a)
    assert shared(9, 1000) == plain(9, 1000) and shared(64, 20000) > plain(64, 20000)
    assert shared(64, 20000, 0) == plain(64, 20000) == shared(64, 20000, 513)      # nothing in common, more groups than are indexed
    try:
        B.set_option(B.OPT_DECODE_SHARED, 1)
        assert shared(9, 1000) > plain(9, 1000)
        B.set_option(B.OPT_DECODE_SHARED, 2)
        assert shared(64, 20000) == plain(64, 20000)
    finally:
        B.set_option(B.OPT_DECODE_SHARED, 0)


def test_decode_shared_python_refuses(B):
    ok = dict(q=_z(5, 8, 128), cache=_z(3, 1, 2, 2048), table=_z(5, 2, dtype=I32), lens=_z(5, dtype=I32), off=_z(3, dtype=I32), sh=_z(2, dtype=I32), out=_z(5, 8, 128),
              k=_z(5, 1, 128), v=_z(5, 1, 128), slots=_z(5, dtype=I64), ws=_z(64, dtype=U8), scales=None, scale=0.1)

    def call(**kw):
        a = {**ok, **kw}
        B.decode_shared(a["q"], a["cache"], a["table"], a["lens"], 32, a["off"], a["sh"], a["out"], a["scale"], a["k"], a["v"], a["slots"], a["ws"], kv_scales=a["scales"])
    for kw in ({}, dict(ws=None), dict(k=None, v=None, slots=None), dict(off=_z(1, dtype=I32), sh=_z(0, dtype=I32)), dict(cache=_z(3, 1, 2, 2048, dtype=U8)),
               dict(cache=_z(3, 1, 2, 2048, dtype=U8), scales=_z(3, 1, 2, dtype=F32))):
        with _accepted():
            call(**kw)
    for kw in (dict(off=_z(2, dtype=I32)), dict(off=_z(3, dtype=I64)), dict(sh=_z(2, dtype=I64)), dict(sh=_z(4, dtype=I32)[::2]), dict(off=_z(6, dtype=I32)[::2]), dict(sh=_z(2, 1, dtype=I32)),
               dict(lens=_z(4, dtype=I32)), dict(table=_z(4, 2, dtype=I32)), dict(out=_z(5, 8, 128, dtype=F32)), dict(scales=_z(3, 1, 2, dtype=F32)), dict(slots=_z(4, dtype=I64)),
               dict(ws=_z(128, dtype=U8)[::2]), dict(q=_z(1, 8, 128).expand(5, 8, 128)), dict(lens=_z(5, 1, dtype=I32))):
        with pytest.raises(AssertionError):
            call(**kw)
            pytest.fail(str(kw))
    with pytest.raises(TypeError):
        call(off=None)
