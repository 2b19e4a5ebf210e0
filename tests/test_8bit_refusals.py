"""What the calls for serving in 8 bits refuse: the C ABI by code, before anything is enqueued, and the Python calls by exception (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

BF, F32, U8, I8, I32, I64 = torch.bfloat16, torch.float32, torch.uint8, torch.int8, torch.int32, torch.int64
PTR = 0x10000   # aligned, and never followed: every call below is refused on the host


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    if not binding.is_built():
        import __graft_entry__
        __graft_entry__.build()
    binding.lib()
    return binding


def _attn(B, **kw):
    a = B.Attn(num_q_heads=8, num_kv_heads=1, head_dim=128, dtype=B.BF16, block_size=16, num_blocks=64, max_blocks_per_seq=8, softmax_scale=0.1,
               kv_format=B.KV_FP8_E4M3_BLOCKS)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _calls(B, a, scales=PTR, ws=PTR, ws_bytes=1 << 30):
    """Every call over a cache with block scales, for one sequence of one token."""
    L, r = B.lib(), ctypes.byref(a)
    return [L.shiftattn_kv_write_scaled(PTR, PTR, PTR, 1, PTR, scales, r, None),
            L.shiftattn_prefill_scaled(PTR, None, None, None, PTR, scales, PTR, PTR, PTR, 1, 1, 1, 1, PTR, ws, ws_bytes, r, None),
            L.shiftattn_decode_scaled(PTR, None, None, None, PTR, scales, PTR, PTR, 1, 1, PTR, ws, ws_bytes, r, None),
            L.shiftattn_mixed_scaled(PTR, None, None, None, PTR, scales, PTR, PTR, PTR, 1, 1, 1, 1, 1, 1, PTR, ws, ws_bytes, r, None)]


def test_the_scaled_calls_want_scales_and_their_format(B):
    assert _calls(B, _attn(B), scales=None) == [B.EINVAL] * 4 and "kv_scales" in B.last_error()
    assert _calls(B, _attn(B), scales=PTR + 4) == [B.EINVAL] * 4
    for fmt in (B.KV_SAME, B.KV_FP8_E4M3, 3, -1):
        assert _calls(B, _attn(B, kv_format=fmt, k_scale=1.0, v_scale=1.0)) == [B.EINVAL] * 4
    assert _calls(B, _attn(B, head_dim=120)) == [B.EUNSUPPORTED] * 4      # not a multiple of 16
    assert _calls(B, _attn(B, block_size=32)) == [B.EUNSUPPORTED] * 4
    assert _calls(B, _attn(B, kv_stride=64)) == [B.EINVAL] * 4
    assert _calls(B, _attn(B, reserved=1)) == [B.EINVAL] * 4
    assert _calls(B, _attn(B), ws=None, ws_bytes=0)[1:] == [B.EWORKSPACE] * 3
    assert _calls(B, _attn(B), ws_bytes=16)[1:] == [B.EWORKSPACE] * 3


def test_the_other_calls_refuse_a_cache_with_block_scales(B):
    L, r = B.lib(), ctypes.byref(_attn(B))
    assert L.shiftattn_kv_write(PTR, PTR, PTR, 1, PTR, r, None) == B.EINVAL and "_scaled" in B.last_error()
    assert L.shiftattn_prefill(PTR, None, None, None, PTR, PTR, PTR, PTR, 1, 1, 1, 1, PTR, PTR, 1 << 30, r, None) == B.EINVAL
    assert L.shiftattn_decode(PTR, None, None, None, PTR, PTR, PTR, 1, 1, PTR, PTR, 1 << 30, r, None) == B.EINVAL
    assert L.shiftattn_decode_static(PTR, None, None, None, PTR, PTR, PTR, 1, 1, PTR, r, None) == B.EINVAL
    assert L.shiftattn_mixed(PTR, None, None, None, PTR, PTR, PTR, PTR, 1, 1, 1, 1, 1, 1, PTR, PTR, 1 << 30, r, None) == B.EINVAL


def test_workspace_sizes_and_plans_take_the_format(B):
    a, f = _attn(B, max_blocks_per_seq=2000), _attn(B, max_blocks_per_seq=2000, kv_format=B.KV_FP8_E4M3, k_scale=1.0, v_scale=1.0)
    assert B.decode_workspace_bytes(8, 4000, a) == B.decode_workspace_bytes(8, 4000, f) > 0
    assert B.prefill_workspace_bytes(2, 2000, 1000, 17000, a) >= 2 * 17000 * 2 * 128 * 2      # the widened cache, at least
    assert B.mixed_workspace_bytes(1, 1000, 1000, 21000, 97, 16000, a) > 0
    plan = B.prefill_plan(1, 1000, 1000, 21000, a, 97, 16000)
    assert plan.decode_wgs > 0 and plan.wave_columns == 32                                   # one launch, the kernel that follows the maximum
    assert B.prefill_plan(1, 16384, 16384, 16384, _attn(B)).wave_columns == 32
    for kw in (dict(head_dim=64), dict(dtype=B.F32)):
        assert B.decode_workspace_bytes(8, 4000, _attn(B, **kw)) == 0 == B.prefill_workspace_bytes(2, 2000, 1000, 17000, _attn(B, **kw))
    assert B.lib().shiftattn_decode_workspace_bytes(8, 4000, ctypes.byref(_attn(B, head_dim=24))) == ctypes.c_size_t(-1).value


def _z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


def _accepted():
    """Any call's arguments are fine but for the place they are in: the last thing asked about."""
    return pytest.raises(RuntimeError, match="a tensor on the GPU is wanted")


SCALES = [_z(3, 1, 2), _z(3, 2, 2, dtype=F32), _z(4, 1, 2, dtype=F32), _z(3, 1, 1, dtype=F32), _z(3, 2, dtype=F32), _z(3, 1, 4, dtype=F32)[..., ::2]]


def _each_call(B, cache, scales):
    q, k, slots, lens = _z(5, 4, 64), _z(5, 1, 64), _z(5, dtype=I64), _z(5, dtype=I32)
    new = dict(k_new=k, v_new=k, slot_mapping=slots, workspace=_z(64, dtype=U8), kv_scales=scales)
    yield lambda: B.kv_write(k, k, slots, cache, kv_scales=scales)
    yield lambda: B.attn_desc(q, cache, _z(5, 2, dtype=I32), 0.1, kv_scales=scales)
    yield lambda: B.prefill(q, cache, _z(2, 2, dtype=I32), _z(3, dtype=I32), lens[:2], 3, 32, q, 0.1, **new)
    yield lambda: B.decode(q, cache, _z(5, 2, dtype=I32), lens, 32, q, 0.1, **new)
    yield lambda: B.mixed(q, cache, _z(2, 2, dtype=I32), _z(2, dtype=I32), lens[:2], 1, 4, 32, 32, q, 0.1, **new)


def test_python_calls_take_scales_that_fit_the_cache(B):
    good = _z(3, 1, 2, 1024, dtype=U8)
    for i, call in enumerate(_each_call(B, good, _z(3, 1, 2, dtype=F32))):
        if i == 1:
            assert call().kv_format == B.KV_FP8_E4M3_BLOCKS
        else:
            with _accepted():
                call()
    for scales in SCALES:
        for call in _each_call(B, good, scales):
            with pytest.raises(AssertionError, match="kv_scales"):
                call()
    for call in _each_call(B, _z(3, 1, 2, 1024), _z(3, 1, 2, dtype=F32)):      # a bf16 cache has none
        with pytest.raises(AssertionError, match="kv_scales"):
            call()
    for call in _each_call(B, good, np.zeros((3, 1, 2), np.float32)):
        with pytest.raises(TypeError):
            call()


# ---- tables -------------------------------------------------------------------------------------------------------------
def _tables(B, **kw):
    t = B.Tables(num_seqs=3, max_blocks_per_seq=4, num_blocks=9, reserved=0, seq_lens=PTR, block_table=PTR, free_blocks=PTR, free_count=PTR)
    for k, v in kw.items():
        setattr(t, k, v)
    return ctypes.byref(t)


def test_tables_calls_refuse(B):
    L, need = B.lib(), B.tables_workspace_bytes(3)
    assert need > 0 and L.shiftattn_tables_workspace_bytes(-1) == ctypes.c_size_t(-1).value
    append = lambda t, new=PTR, pre=1, total=5, rows=7, cu=PTR, slots=PTR, taken=PTR, ws=PTR, n=need: L.shiftattn_tables_append(t, new, pre, total, rows, cu, slots, taken, ws, n, None)
    cut = lambda t, keep=PTR, ws=PTR, n=need: L.shiftattn_tables_truncate(t, keep, ws, n, None)
    for kw in (dict(num_seqs=-1), dict(max_blocks_per_seq=-1), dict(num_blocks=-1), dict(reserved=1), dict(seq_lens=None), dict(block_table=None),
               dict(free_blocks=None), dict(free_count=None), dict(seq_lens=PTR + 2), dict(free_count=PTR + 1)):
        assert append(_tables(B, **kw)) == B.EINVAL and cut(_tables(B, **kw)) == B.EINVAL, kw
    assert append(None) == B.EINVAL and cut(None) == B.EINVAL
    t = _tables(B)
    for kw in (dict(pre=4), dict(pre=-1), dict(total=-1), dict(rows=-1), dict(rows=6), dict(total=2 ** 31 - 1, rows=2 ** 31 - 1), dict(new=None), dict(cu=None),
               dict(slots=None), dict(taken=None), dict(slots=PTR + 4), dict(cu=PTR + 2)):
        assert append(t, **kw) == B.EINVAL, kw
    assert cut(t, keep=None) == B.EINVAL
    for kw in (dict(ws=None), dict(n=need - 1), dict(ws=PTR + 2)):
        assert append(t, **kw) == B.EWORKSPACE and cut(t, **kw) == B.EWORKSPACE
    assert cut(_tables(B, num_seqs=0)) == B.OK


def test_python_tables_calls_refuse(B):
    i = lambda *s: _z(*s, dtype=I32)
    good = dict(new=i(3), pre=1, total=5, lens=i(3), table=i(3, 4), free=i(9), count=i(1), cu=i(2), slots=_z(7, dtype=I64), taken=i(3), ws=_z(64, dtype=U8))

    def append(**kw):
        a = {**good, **kw}
        B.tables_append(a["new"], a["pre"], a["total"], a["lens"], a["table"], a["free"], a["count"], a["cu"], a["slots"], a["taken"], workspace=a["ws"])

    def cut(**kw):
        a = {**good, **kw}
        B.tables_truncate(a["new"], a["lens"], a["table"], a["free"], a["count"], workspace=a["ws"])
    for call in (append, cut):
        for ws in (good["ws"], None):
            with _accepted():
                call(ws=ws)
        for kw in (dict(new=i(4)), dict(new=_z(3, dtype=I64)), dict(lens=i(2)), dict(lens=_z(3, dtype=I64)), dict(table=i(2, 4)), dict(table=i(3, 8)[:, ::2]),
                   dict(table=_z(3, 4, dtype=I64)), dict(free=i(3, 3)), dict(free=_z(9, dtype=I64)), dict(count=i(2)), dict(count=_z(1, dtype=I64)),
                   dict(new=i(6)[::2]), dict(ws=_z(128, dtype=U8)[::2])):
            with pytest.raises(AssertionError):
                call(**kw)
        with pytest.raises(ValueError):
            call(table=i(12))
    for kw in (dict(cu=i(3)), dict(cu=_z(2, dtype=I64)), dict(pre=2), dict(slots=i(7)), dict(slots=_z(14, dtype=I64)[::2]), dict(taken=i(2)),
               dict(taken=_z(3, dtype=I64))):
        with pytest.raises(AssertionError):
            append(**kw)


# ---- int8 ---------------------------------------------------------------------------------------------------------------
def test_int8_calls_refuse(B):
    L = B.lib()
    x = lambda **kw: ctypes.byref(B.Xchg(**{**dict(P=1, num_q_heads=8, num_kv_heads=1, head_dim=128, dtype=B.BF16), **kw}))
    qkv = lambda d=512, xc=None, T=3, Tp=4, p=PTR, s=PTR, ws=None, n=0: L.shiftattn_qkv_proj_pack_int8_ws(p, s, PTR, PTR, PTR, T, Tp, d, xc or x(), ws, n, None)
    o = lambda d=512, xc=None, T=3, Tp=4, p=PTR, s=PTR, ws=None, n=0: L.shiftattn_unpack_o_proj_int8_ws(p, s, PTR, PTR, PTR, T, Tp, d, xc or x(), ws, n, None)
    for call in (qkv, o):
        assert call(T=5, Tp=4) == B.EINVAL and call(T=-1) == B.EINVAL and call(d=0) == B.EINVAL
        assert call(p=None) == B.EINVAL and call(s=None) == B.EINVAL and call(p=PTR + 8) == B.EINVAL and call(s=PTR + 2) == B.EINVAL
        assert call(n=16) == B.EINVAL and call(ws=PTR + 8, n=16) == B.EINVAL
        assert call(d=100) == B.EUNSUPPORTED and call(xc=x(head_dim=64)) == B.EUNSUPPORTED and call(xc=x(dtype=B.F32)) == B.EUNSUPPORTED
    # sums of products stay below 2^31
    assert qkv(d=131072) == B.EUNSUPPORTED and "131072" in B.last_error()
    assert o(xc=x(num_q_heads=1024)) == B.EUNSUPPORTED
    for f in (L.shiftattn_quantize_rows_int8,):
        assert f(PTR, PTR, PTR, -1, 8, None) == B.EINVAL and f(PTR, PTR, PTR, 1, 12, None) == B.EUNSUPPORTED
        assert f(None, PTR, PTR, 1, 8, None) == B.EINVAL and f(PTR, PTR + 4, PTR, 1, 8, None) == B.EINVAL and f(PTR, PTR, PTR, 0, 8, None) == B.OK
    assert L.shiftattn_quantize_recv_int8(PTR, PTR, PTR, 1, 1, x(dtype=B.F32), None) == B.EUNSUPPORTED
    assert L.shiftattn_quantize_recv_int8(PTR + 8, PTR, PTR, 1, 1, x(), None) == B.EINVAL


def test_int8_workspace_is_that_of_fp8_codes(B):
    for shape in ((1, 2304, 16384), (48, 1280, 8192), (300, 10240, 8192), (0, 256, 256)):
        assert B.proj_workspace_bytes_int8(*shape) == B.proj_workspace_bytes(*shape, fp8=True)


def test_python_int8_calls_refuse(B):
    c = lambda *s: _z(*s, dtype=I8)
    f = lambda *s: _z(*s, dtype=F32)
    with _accepted():
        B.quantize_rows_int8(_z(4, 64), c(4, 64), f(4))
    for args in ((_z(4, 64), _z(4, 64, dtype=U8), f(4)), (_z(4, 64), c(4, 64), f(5)), (f(4, 64), c(4, 64), f(4)), (_z(4, 64), c(4, 32), f(4)),
                 (_z(4, 128)[:, ::2], c(4, 64), f(4))):
        with pytest.raises(AssertionError):
            B.quantize_rows_int8(*args)
    with _accepted():
        B.quantize_recv_int8(_z(1, 4, 2, 128), c(1, 4, 2, 128), f(4))
    for args in ((_z(1, 4, 2, 128), _z(1, 4, 2, 128, dtype=U8), f(4)), (_z(1, 4, 2, 128), c(1, 4, 2, 64), f(4)), (f(1, 4, 2, 128), c(1, 4, 2, 128), f(4))):
        with pytest.raises(AssertionError):
            B.quantize_recv_int8(*args)
    for ws in (None, _z(64, dtype=U8)):
        with _accepted():
            B.qkv_proj_pack_int8(c(4, 256), f(4), c(768, 256), f(768), _z(1, 4, 6, 128), 1, 4, 1, ws)
        with _accepted():
            B.unpack_o_proj_int8(c(1, 4, 2, 128), f(4), c(256, 256), f(256), _z(4, 256), ws)
    u = lambda *s: _z(*s, dtype=U8)
    for args in ((u(4, 256), f(4), u(768, 256), f(768), _z(1, 4, 6, 128)), (c(4, 256), f(3), c(768, 256), f(768), _z(1, 4, 6, 128)),
                 (c(4, 256), f(4), c(768, 128), f(768), _z(1, 4, 6, 128)), (c(4, 256), f(4), c(768, 256), f(768), f(1, 4, 6, 128)),
                 (c(4, 256), f(4), c(768, 256), f(768), _z(1, 4, 5, 128))):
        with pytest.raises(AssertionError):
            B.qkv_proj_pack_int8(*args, 1, 4, 1)
    for args in ((u(1, 4, 2, 128), f(4), u(256, 256), f(256), _z(4, 256)), (c(1, 4, 2, 128), f(3), c(256, 256), f(256), _z(4, 256)),
                 (c(1, 4, 2, 128), f(4), c(256, 128), f(256), _z(4, 256)), (c(1, 4, 2, 128), f(4), c(256, 256), f(255), _z(4, 256))):
        with pytest.raises(AssertionError):
            B.unpack_o_proj_int8(*args)
    with pytest.raises(AssertionError):   # and the FP8 calls int8 codes
        B.quantize_rows_fp8(_z(4, 64), c(4, 64), f(4))
