"""Residual addition and norm against its definition: values, codes, scales and the stream itself bit for bit (sums are in 64 bits, so
their order decides nothing)."""
import numpy as np
import pytest

import plain_8bit as P
import plain_layer as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _dev(a, kind):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV, {"bf16": torch.bfloat16, "f32": torch.float32}[kind])


def _np(t):
    import torch
    torch.cuda.synchronize()
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def _same(got, want, what):
    assert got.shape == want.shape
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all() and (got[~nan] == want[~nan]).all(), what


def _values(rng, shape, kind, spread=0.7):
    x = (rng.standard_normal(shape) * np.exp(spread * rng.standard_normal((shape[0], 1)))).astype(np.float32)
    return P.bf16(x) if kind == "bf16" else x


def _run(B, x, res, w, kinds, out_kind, offset=0.0, pad=0):
    """Through the call; pad > 0: rows of wider tensors, whose other columns have to stay."""
    import torch
    rows, cols = x.shape
    wide = lambda t: t if not pad else torch.cat([t, torch.full((rows, pad), 3, dtype=t.dtype, device=DEV)], 1)
    xd, rd = wide(_dev(x, kinds[0])), None if res is None else wide(_dev(res, kinds[1]))
    out = wide(torch.full((rows, cols), 7, dtype={"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.uint8, "int8": torch.int8}[out_kind], device=DEV))
    scales = torch.full((rows,), -1.0, device=DEV) if out_kind in ("fp8", "int8") else None
    cut = lambda t: None if t is None else t[:, :cols]
    B.add_rms_norm(cut(xd), _dev(w, kinds[2]), cut(out), EPS, residual=cut(rd), scales=scales, weight_offset=offset)
    if pad:
        assert all((_np(t)[:, cols:] == 3).all() for t in (xd, rd, out) if t is not None)
    return _np(cut(out)), None if rd is None else _np(cut(rd)), None if scales is None else _np(scales)


def _check(got, x, res, w, kinds, out_kind, offset):
    y, h = L.rms_norm_rows(x, res, w, EPS, offset, kinds[1] == "bf16")
    out, stream, scales = got
    if res is not None:
        _same(stream, h, "residual")
    if out_kind == "f32":
        _same(out, y, "out")
    elif out_kind == "bf16":
        _same(out, P.bf16(y), "out")
    else:
        codes, want = (L.fp8_rows if out_kind == "fp8" else L.int8_rows)(y)
        _same(scales, want, "scales")
        if out_kind == "fp8":
            nan = codes & 0x7F == 0x7F
            assert ((out & 0x7F == 0x7F) == nan).all() and (out[~nan] == codes[~nan]).all()
        else:
            assert (out == codes).all()


OUT = ["bf16", "f32", "fp8", "int8"]


@pytest.mark.parametrize("out_kind", OUT)
@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 8192), (3, 64), (7, 136), (5, 1000), (19, 2048), (4, 4104), (9, 5120), (2, 8200), (2, 16384), (1, 40000), (2, 65536), (2100, 512)])
def test_sizes(B, rows, cols, out_kind):
    rng = np.random.Generator(np.random.PCG64(rows * 70001 + cols))
    x, res, w = _values(rng, (rows, cols), "bf16"), _values(rng, (rows, cols), "bf16"), P.bf16(1 + 0.3 * rng.standard_normal(cols).astype(np.float32))
    kinds = ("bf16", "bf16", "bf16")
    _check(_run(B, x, res, w, kinds, out_kind), x, res, w, kinds, out_kind, 0.0)


@pytest.mark.parametrize("out_kind", OUT)
@pytest.mark.parametrize("kinds", [("bf16", "f32", "bf16"), ("f32", "f32", "f32"), ("f32", "bf16", "bf16"), ("bf16", None, "bf16"), ("f32", None, "f32")])
@pytest.mark.parametrize("cols,pad,offset", [(5120, 0, 0.0), (264, 16, 1.0), (24, 8, -0.5)])
def test_types_strides_and_weights_from_one(B, kinds, out_kind, cols, pad, offset):
    rng = np.random.Generator(np.random.PCG64(cols + len(str(kinds))))
    x, w = _values(rng, (5, cols), kinds[0]), _values(rng, (1, cols), kinds[2])[0]
    res = None if kinds[1] is None else _values(rng, (5, cols), kinds[1], 2.0)
    _check(_run(B, x, res, w, kinds, out_kind, offset, pad), x, res, w, kinds, out_kind, offset)


@pytest.mark.parametrize("out_kind", OUT)
def test_rows_of_zeros_infinities_nan_and_far_magnitudes(B, out_kind):
    rng = np.random.Generator(np.random.PCG64(5))
    cols = 520
    x = _values(rng, (12, cols), "f32")
    x[1] = 0
    x[2, 7] = np.nan
    x[3, 100] = np.inf
    x[4, 3], x[4, 5] = np.inf, -np.inf
    x[5] *= np.float32(1e30)
    x[6] *= np.float32(1e-30)
    x[7] = 0
    x[7, 519] = 1e-20
    x[8] = np.float32(3e38)
    x[9] *= np.float32(1e-42) / np.abs(x[9]).max()
    w = _values(rng, (1, cols), "f32")[0]
    w[11] = 0
    kinds = ("f32", "f32", "f32")
    _check(_run(B, x, None, w, kinds, out_kind), x, None, w, kinds, out_kind, 0.0)
    w[40] = np.inf                                          # the weights' own
    w[41] = np.nan
    _check(_run(B, x[:2], None, w, kinds, out_kind), x[:2], None, w, kinds, out_kind, 0.0)


@pytest.mark.parametrize("residual", [False, True])
def test_the_output_may_be_the_input(B, residual):
    import torch
    rng = np.random.Generator(np.random.PCG64(6))
    x, res, w = _values(rng, (6, 4096), "bf16"), _values(rng, (6, 4096), "bf16") if residual else None, _values(rng, (1, 4096), "bf16")[0]
    xd, rd = _dev(x, "bf16"), _dev(res, "bf16") if residual else None
    B.add_rms_norm(xd, _dev(w, "bf16"), xd, EPS, residual=rd)
    y, h = L.rms_norm_rows(x, res, w, EPS)
    _same(_np(xd), P.bf16(y), "out")
    if residual:
        _same(_np(rd), h, "residual")
    both = _dev(x, "bf16")                                  # a row added to itself
    out = torch.empty_like(both)
    B.add_rms_norm(both, _dev(w, "bf16"), out, EPS, residual=both)
    y, h = L.rms_norm_rows(x, x, w, EPS)
    _same(_np(both), h, "residual")
    _same(_np(out), P.bf16(y), "out")


def test_many_rows_of_any_length(B):
    rng = np.random.Generator(np.random.PCG64(8))
    x, res, w = _values(rng, (70001, 16), "bf16"), _values(rng, (70001, 16), "bf16"), _values(rng, (1, 16), "bf16")[0]
    kinds = ("bf16", "bf16", "bf16")
    for out_kind in ("bf16", "int8"):
        _check(_run(B, x, res, w, kinds, out_kind), x, res, w, kinds, out_kind, 0.0)


def test_codes_are_those_of_the_quantisers_of_a_row_in_32_bits(B):
    """Where y is a bf16 value the quantisers of bf16 rows give the same codes and scales."""
    import torch
    rng = np.random.Generator(np.random.PCG64(9))
    x = rng.choice(np.array([-1, 1], np.float32), (33, 1024))          # rms 1: inv is a power of two's neighbour, the same for all elements
    w = P.bf16(rng.standard_normal(1024).astype(np.float32))
    y32 = torch.empty((33, 1024), device=DEV)
    B.add_rms_norm(_dev(x, "bf16"), _dev(w, "bf16"), y32, 2.0 ** -60)
    assert (_np(y32) == x * w).all()
    for name, dtype in (("fp8", torch.uint8), ("int8", torch.int8)):
        codes, scales = torch.empty((33, 1024), dtype=dtype, device=DEV), torch.empty(33, device=DEV)
        B.add_rms_norm(_dev(x, "bf16"), _dev(w, "bf16"), codes, 2.0 ** -60, scales=scales)
        c2, s2 = torch.empty_like(codes), torch.empty_like(scales)
        getattr(B, "quantize_rows_" + name)(y32.to(torch.bfloat16), c2, s2)
        assert torch.equal(codes, c2) and torch.equal(scales, s2), name
