"""The plain implementations that the 8-bit operators are held to, against definitions and other implementations (no GPU)."""
import numpy as np
import pytest

import plain_8bit as P


def test_e4m3_codes_agree_with_the_oracle(oracle):
    rng = np.random.Generator(np.random.PCG64(1))
    x = np.concatenate([rng.standard_normal(2000) * 10.0 ** rng.uniform(-5, 3, 2000), P.e4m3_values()[:0x7F], -P.e4m3_values()[:0x7F],
                        (P.e4m3_values()[:0x7E] + P.e4m3_values()[1:0x7F]) / 2, [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 464, 1e9, -np.inf]])
    x = x.astype(np.float32)
    with np.errstate(invalid="ignore"):
        assert P.e4m3_codes(x.astype(np.float64)).tolist() == [oracle.e4m3_from_float(float(v)) for v in np.clip(x, -448, 448)]
    assert all(P.e4m3_values()[c] == oracle.e4m3_value(c) for c in range(256) if c & 0x7F != 0x7F)


def test_scales_are_the_least_that_hold_the_values():
    for top in (1e-40, 2.0 ** -100, 448 * 2.0 ** -100, 0.3, 1.75, np.nextafter(np.float32(1.75), np.float32(2)), 448, 449, 3e38):
        s = P.needed(np.array([0.0, -top]))
        assert 2.0 ** P.E_MIN <= s <= 2.0 ** P.E_MAX
        assert top <= 448 * s or s == 2.0 ** P.E_MAX
        assert s == 2.0 ** P.E_MIN or top > 448 * s / 2
    assert P.needed(np.array([np.inf, np.nan, 1.0])) == P.needed(np.array([1.0])) and P.needed(np.array([np.inf])) == 2.0 ** P.E_MIN


@pytest.mark.parametrize("steps", [[16], [1] * 16, [5, 1, 1, 9], [16, 16, 7]])
def test_appends_keep_what_the_format_can(steps):
    """However a block is filled, a stored value is within half a step of the final scale (twice: it may have been rounded before)."""
    rng = np.random.Generator(np.random.PCG64(2))
    n, D = sum(steps), 32
    x = rng.standard_normal((n, 1, D)).astype(np.float32) * np.exp(rng.standard_normal((n, 1, 1))).astype(np.float32)
    c = P.Cache(2 + n // 16, 1, D, rng)
    at = 0
    for k in steps:
        c.append(x[at:at + k], -x[at:at + k], np.arange(at, at + k))
        at += k
    got = c.rows(np.arange(1 + n // 16), n, 0, 0)
    s = np.repeat(c.scales[:, 0, 0], 16)[:n, None]
    tol = np.maximum(np.abs(x[:, 0]) * 2.0 ** -4, s * 2.0 ** -10) * (1 if len(steps) == 1 else 2)
    assert np.all(np.abs(got - x[:, 0]) <= tol)
    assert np.array_equal(c.rows(np.arange(1 + n // 16), n, 0, 1), -got)


def test_tables_append_and_truncate_are_inverse():
    rng = np.random.Generator(np.random.PCG64(3))
    t = P.Tables([0] * 9, 40, rng.permutation(200), 200)
    t.append([100, 0, 33, 1, 1, 0, 1, 1, 1], 3, 133, 140)
    before = t.lens.copy(), t.free[:t.count].copy(), t.count
    cu, slots, taken = t.append([7, 40, 0, 1, 1, 1, 0, 1, 1], 3, 50, 60)
    assert cu.tolist() == [0, 7, 47, 47] and taken.tolist() == [7, 40, 0, 1, 1, 1, 0, 1, 1]
    used = slots[slots >= 0]
    assert len(set(used.tolist())) == len(used) == taken.sum() and np.all(slots[47:50] == -1) and slots[50 + 3] == -1
    held = [t.table[s, b] for s in range(9) for b in range(-(-int(t.lens[s]) // 16))]
    assert sorted(held + t.free[:t.count].tolist()) == list(range(200))
    t.truncate(before[0])
    assert np.array_equal(t.lens, before[0]) and t.count == before[2] and np.array_equal(t.free[:t.count], before[1])


def test_tables_refuse_in_order():
    t = P.Tables([0, 0, 0, 0, 0], 4, np.arange(5), 5)
    cu, slots, taken = t.append([64, 65, 33, 1, 2], 3, 200, 210)   # 4 blocks; too long; 3 blocks of one left; one; two tokens in one row
    assert taken.tolist() == [64, 0, 0, 0, 0] and cu.tolist() == [0, 64, 64, 64] and t.count == 1
    t = P.Tables([0, 0, 15], 4, np.arange(5), 2)
    cu, slots, taken = t.append([20, 20, 1], 2, 30, 31)            # rows run out at the second; the third needs no block
    assert taken.tolist() == [20, 0, 1] and t.count == 0


def test_int8_codes_are_within_half_a_step():
    rng = np.random.Generator(np.random.PCG64(4))
    x = P.bf16(rng.standard_normal((7, 200)) * 10.0 ** rng.integers(-30, 30, (7, 1)))
    x[3] = 0
    c, s = P.quantise_int8(x)
    assert np.abs(c).max() <= 127 and s[3] == 1 and not c[3].any()
    assert np.all(np.abs(c * s[:, None].astype(np.float64) - x) <= s[:, None] * 0.50001)
