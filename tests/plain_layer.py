"""Plain numpy forms of the operators around a layer's projections, from their definitions: what the kernels' results are compared with."""
import numpy as np

import plain_8bit as P


def rms_norm_rows(x, residual, weight, eps, offset=0.0, residual_bf16=True):
    """(y in float32, what the residual becomes) of float32 arrays that hold bf16 or float32 values: every operation as the library defines
    it, so that the bits are the library's."""
    with np.errstate(all="ignore"):
        h = np.asarray(x, np.float32)
        if residual is not None:
            h = h + np.asarray(residual, np.float32)
            if residual_bf16:
                h = P.bf16(h)
        mean = np.square(h.astype(np.float64)).sum(-1, keepdims=True) / h.shape[-1] + np.float64(np.float32(eps))
        inv = (1.0 / np.sqrt(mean)).astype(np.float32)
        return (h * inv) * (np.asarray(weight, np.float32) + np.float32(offset)), h


def fp8_rows(y):
    """(codes, scales) of float32 rows by the rule of quantize_rows_fp8."""
    with np.errstate(all="ignore"):
        top = np.where(np.isnan(y), 0, np.abs(y)).max(-1).astype(np.float32)
        scale = np.where(top > 0, top / np.float32(448), np.float32(1)).astype(np.float32)
        return P.e4m3_codes((y / scale[:, None]).astype(np.float32)), scale


def int8_rows(y):
    """(codes, scales) of float32 rows by the rule of quantize_rows_int8."""
    with np.errstate(all="ignore"):
        top = np.where(np.isfinite(y), np.abs(y), 0).max(-1).astype(np.float32)
        tiny = top < np.float32(2.0 ** -100)
        scale = np.where(tiny, np.float32(1), top * np.float32(1 / 127))
        inv = np.where(tiny, np.float32(1), np.float32(127) * (np.float32(1) / top))
        n = np.rint(np.where(np.isfinite(y), y, 0).astype(np.float64) * inv.astype(np.float64)[:, None])
        codes = np.where(np.isnan(y), 0, np.where(np.isinf(y), np.sign(y) * 127, n))
        return codes.astype(np.int8), scale.astype(np.float32)


def rotary(x, positions, frequencies, pairs=False, magnitude=1.0):
    """[rows, heads, D] in 64 bits; rows with a negative position as they are."""
    x = np.array(x, np.float64)
    half = len(frequencies)
    lo = np.arange(half) * (2 if pairs else 1)
    hi = lo + (1 if pairs else half)
    pos = np.asarray(positions, np.float64)
    t = np.where(pos >= 0, pos, 0)[:, None, None] * np.asarray(frequencies, np.float64)
    a, b = x[..., lo].copy(), x[..., hi].copy()
    there = (pos >= 0)[:, None, None]
    x[..., lo] = np.where(there, magnitude * (a * np.cos(t) - b * np.sin(t)), a)
    x[..., hi] = np.where(there, magnitude * (b * np.cos(t) + a * np.sin(t)), b)
    return x
