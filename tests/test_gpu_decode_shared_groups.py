"""decode_shared where units of shared keys are many and short beside the sequences' own keys: a workgroup takes several of them, of groups of
different length and width, one behind the other (bounds as in test_gpu_decode_shared)."""
import math

import numpy as np
import pytest

import plain_8bit as P
from test_gpu_decode_shared import B, Case

pytestmark = pytest.mark.gpu


def _many(seed, groups, members, pre, suf, empty=0.1):
    rng = np.random.Generator(np.random.PCG64(seed))
    out = []
    for _ in range(groups):
        p = int(rng.integers(16, pre))
        out.append((p if rng.random() > empty else 0, [p + int(n) for n in rng.integers(1, suf, int(rng.integers(0, members + 1)))]))
    return out


@pytest.mark.parametrize("cache", ["same", "fp8", "blocks"])
@pytest.mark.parametrize("groups,hq,hkv", [([(100, [600, 601])] * 64, 32, 8), (_many(1, 90, 4, 900, 700), 16, 4), (_many(2, 500, 2, 200, 300), 8, 1), (_many(3, 30, 20, 300, 500), 16, 8)])
def test_several_units_a_workgroup(B, groups, hq, hkv, cache):
    import torch
    case = Case(groups, [300, 0, 1], hq, hkv, cache=cache, seed=len(groups))
    d, again = case.device(), case.device()
    case.call(B, d)
    case.check(d)
    case.call(B, again)
    torch.cuda.synchronize()
    assert torch.equal(d["out"], again["out"])


@pytest.mark.parametrize("cache", ["same", "fp8"])
@pytest.mark.parametrize("groups", [[(64, [2100, 90]), (1900, [2000, 1990, 2050, 1999]), (48, [100] * 20), (40, [60, 70, 0])] + [(500, [900, 1000])] * 10, [(64, [2100, 1800])] * 30])
def test_groups_that_are_left_alone(B, groups, cache):
    """As calls choose by themselves: groups with little in common share nothing, beside some that do and where there is no other."""
    case = Case(groups, [77, 0], 8, 2, cache=cache, seed=5)
    assert len(case.lens) * int(case.lens.max()) * 2 * 512 // (1 if cache == "same" else 2) > 40e6
    try:
        B.set_option(B.OPT_DECODE_SHARED, 0)
        d = case.device()
        case.call(B, d)
        case.check(d)
    finally:
        B.set_option(B.OPT_DECODE_SHARED, 1)


def test_one_workspace_for_batches_of_any_number_of_groups(B):
    """Sized for the most sequences, tokens and groups, which are the plain kernel's, and taken by every smaller batch."""
    import torch
    cases = [Case([(32, [33 + i % 3, 40]) for i in range(n)], [50], seed=n) for n in (600, 512, 300, 3)]
    ds = [c.device() for c in cases]
    a = B.attn_desc(ds[0]["q"], ds[0]["cache"], ds[0]["table"], cases[0].scale, ds[0]["k"], ds[0]["out"])
    ws = torch.full((B.decode_shared_workspace_bytes(1201, 50, 600, a),), 0xFF, dtype=torch.uint8, device="cuda:0")
    for c, d in zip(cases, ds):
        c.call(B, d, workspace=ws)
        c.check(d)


@pytest.mark.parametrize("members", [2, 20])
@pytest.mark.parametrize("shared", [True, False])
def test_values_of_any_magnitude(B, members, shared):
    """Values times 2^e make outputs times 2^e, to the bit: nothing on the way overflows or loses places where the plain call's sums do not.
    Half of the keys weigh 2^12 times the first ones of every range."""
    import torch
    outs = []
    for e in (0, -100, 100, 115):
        case = Case([(640, [650 + i for i in range(members)])], seed=17)
        case.q[...] = 1
        case.pages[:, :, 0] = 0
        for i in range(40):
            if i // 2 % 2:
                case.pages[case.table[0, i], :, 0] = P.bf16(np.float32(12 * math.log(2) / math.sqrt(128)))
        case.pages[:, :, 1] *= np.float32(2.0 ** e)
        case.v_new *= np.float32(2.0 ** e)
        d = case.device()
        case.call(B, d, shared=shared)
        torch.cuda.synchronize()
        out = d["out"].double() * 2.0 ** -e
        assert torch.isfinite(out).all(), e
        outs.append(out)
    assert all(torch.equal(o, outs[0]) for o in outs)
