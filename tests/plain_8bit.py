"""Plain implementations, in 64 bits on the CPU, of the operators for serving in 8 bits: what their kernels are held to."""
import numpy as np

BLOCK = 16
E_MIN, E_MAX = -100, 119


def bf16(x):
    """Nearest bf16 values of float32 ones, as float32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)


# ---- E4M3 ----------------------------------------------------------------------------------------------------------
def e4m3_values():
    """Value of every code (NaN for 0x7F and 0xFF)."""
    c = np.arange(256)
    m, e, sign = c & 7, (c >> 3) & 15, 1.0 - 2.0 * (c >> 7)
    v = sign * np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    v[[0x7F, 0xFF]] = np.nan
    return v


_VALUES = e4m3_values()


def e4m3_codes(x):
    """Nearest code of doubles, ties to the even code, saturating; NaN to a NaN code of its sign."""
    a = np.minimum(np.abs(x), 448.0)
    e = np.clip(np.frexp(np.where(np.isnan(a), 0, a))[1] - 1, -6, 8)
    step = np.ldexp(1.0, e - 3)
    r = np.round(np.where(np.isnan(a), 0, a) / step) * step          # numpy rounds ties to even: multiples of the step are codes in order
    code = np.searchsorted(_VALUES[:0x7F], r)
    code = np.where(np.isnan(x), 0x7F, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


# ---- the cache with block scales ---------------------------------------------------------------------------------------
def needed(x):
    """Scale that a block of values wants."""
    x = np.abs(x[np.isfinite(x)])
    top = float(x.max()) if x.size else 0.0
    e = E_MIN
    while e < E_MAX and top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """codes [num_blocks, heads, 2, 16 D] uint8 and scales [num_blocks, heads, 2]."""

    def __init__(self, num_blocks, heads, D, rng=None):
        self.D, self.heads = D, heads
        self.codes = np.zeros((num_blocks, heads, 2, BLOCK * D), np.uint8)
        self.scales = np.zeros((num_blocks, heads, 2), np.float32)
        if rng is not None:   # what earlier owners of the blocks left
            self.codes[:] = rng.integers(0, 256, self.codes.shape)
            self.scales[:] = 2.0 ** rng.integers(-8, 9, self.scales.shape)

    def part(self, blk, g, x):
        """The codes of one block, head and part as [token, d] (a view)."""
        p = self.codes[blk, g, x]
        return p.reshape(BLOCK, self.D) if x == 0 else p.reshape(self.D, BLOCK).T

    def append(self, k, v, slots):
        """k, v [tokens, heads, D] float32."""
        i, n = 0, len(slots)
        while i < n:
            if slots[i] < 0:
                i += 1
                continue
            j = i + 1
            while j < n and slots[j] == slots[j - 1] + 1 and slots[j] % BLOCK:
                j += 1
            blk, o = divmod(int(slots[i]), BLOCK)
            for g in range(self.heads):
                for x, rows in enumerate((k, v)):
                    new = rows[i:j, g].astype(np.float64)
                    s = needed(new)
                    at = self.part(blk, g, x)
                    if o:
                        had = float(self.scales[blk, g, x])
                        if s > had:
                            at[:o] = e4m3_codes(_VALUES[at[:o]] * (had / s))
                        s = max(s, had)
                    with np.errstate(over="ignore"):
                        at[o:o + j - i] = e4m3_codes(new / s)
                    self.scales[blk, g, x] = s
            i = j

    def rows(self, table, length, g, x):
        """Values of a sequence's first `length` tokens: [length, D] doubles."""
        out = np.zeros((length, self.D))
        for b in range(-(-length // BLOCK)):
            n = min(BLOCK, length - b * BLOCK)
            out[b * BLOCK:b * BLOCK + n] = _VALUES[self.part(table[b], g, x)[:n]] * float(self.scales[table[b], g, x])
        return out


def attend(q, cache, table, length, scale):
    """q [n, hq, D]: the last n tokens of a sequence of `length`.  Returns the result and, for bounds on its error, the sum of
    p |v| and the largest sum of |q||k| scale that meets a row: [n, hq, D], [n, hq, D], [n, hq, 1]."""
    n, hq, D = q.shape
    G = hq // cache.heads
    out, mag, big = np.zeros((n, hq, D)), np.zeros((n, hq, D)), np.zeros((n, hq, 1))
    hidden = np.arange(length) > np.arange(length - n, length)[:, None]
    for g in range(cache.heads):
        k, v = cache.rows(table, length, g, 0), cache.rows(table, length, g, 1)
        for j in range(g * G, g * G + G):
            s = np.where(hidden, -np.inf, (q[:, j].astype(np.float64) @ k.T) * scale)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            out[:, j], mag[:, j] = p @ v, p @ np.abs(v)
            big[:, j, 0] = np.where(hidden, 0, np.abs(q[:, j].astype(np.float64)) @ np.abs(k).T).max(1) * scale
    return out, mag, big


def bound(dtype, out, mag, big, D, keys):
    """How far a result may be off.  bf16: the probabilities and the result are each rounded to bf16 (2^-8 of their value at most), and
    the logits' float32 sums of D products move a probability by D 2^-24 of the largest sum of magnitudes, twice (its own and the
    sum's).  fp32: the same without the bf16 roundings, and a sum over the keys."""
    logits = 2.0 ** -24 * (2 * (D + 4) * big + 16)
    if dtype == "f32":
        return mag * (logits + keys * 2.0 ** -24) + 1e-30
    return 2.0 ** -8 * (mag + np.abs(out)) + mag * (logits + keys * 2.0 ** -24) + 1e-30


# ---- tables --------------------------------------------------------------------------------------------------------------
class Tables:
    def __init__(self, lens, max_blocks, free, count):
        self.lens, self.free, self.count, self.max_blocks = np.array(lens, np.int32), np.array(free, np.int32), int(count), max_blocks
        self.table = np.full((len(lens), max_blocks), -1, np.int32)

    def append(self, new, num_prefill, total, rows):
        """cu, slots, taken; lens, table and count move on."""
        taken, slots, cu = [], np.full(rows, -1, np.int64), [0]
        asked = needed = 0
        height = min(max(self.count, 0), len(self.free))
        for s in range(len(self.lens)):
            had, n, chunk = max(int(self.lens[s]), 0), max(int(new[s]), 0), s < num_prefill
            ok = had + n <= BLOCK * self.max_blocks and (chunk or n <= 1)
            if ok and chunk:
                asked += n
                ok = asked <= total
            take = 0
            if ok:
                first, last = -(-had // BLOCK), -(-(had + n) // BLOCK)
                needed += last - first
                if first == last or needed <= height:
                    take = n
                    for b in range(first, last):
                        self.table[s, b] = self.free[height - 1 - (needed - (last - first)) - (b - first)]
                    self.count = height - needed if first != last else self.count
            row = cu[-1] if chunk else total + s - num_prefill
            for i in range(take):
                slots[row + i] = int(self.table[s, (had + i) // BLOCK]) * BLOCK + (had + i) % BLOCK
            if take:
                self.lens[s] = had + take
            if chunk:
                cu.append(cu[-1] + take)
            taken.append(take)
        self.count = min(max(self.count, 0), len(self.free))
        return np.array(cu, np.int32), slots, np.array(taken, np.int32)

    def truncate(self, keep):
        back = []
        for s, k in enumerate(keep):
            if 0 <= k < self.lens[s]:
                back += [self.table[s, b] for b in range(-(-int(k) // BLOCK), -(-int(self.lens[s]) // BLOCK))]
                self.lens[s] = k
        for b in reversed(back):
            self.free[self.count] = b
            self.count += 1


# ---- int8 ------------------------------------------------------------------------------------------------------------------
def quantise_int8(x):
    """Rows of float32 (bf16) values: int8 codes and float32 scales."""
    x = np.asarray(x, np.float32)
    top = np.where(np.isfinite(x), np.abs(x), 0).max(-1, keepdims=True).astype(np.float32)
    tiny = top < np.float32(2.0 ** -100)
    safe = np.where(tiny, np.float32(1), top)
    inv, scale = np.where(tiny, np.float32(1), np.float32(127) * (np.float32(1) / safe)), np.where(tiny, np.float32(1), safe * (np.float32(1) / np.float32(127)))
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.clip(np.round(x.astype(np.float64) * inv), -127, 127)
    return np.where(np.isnan(y), 0, y).astype(np.int8), scale[..., 0]
