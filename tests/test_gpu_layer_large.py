"""The operators around the projections and decode_shared where counts and offsets pass 32 bits: rows beyond one launch, caches beyond 4 GiB."""
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


def test_more_rows_than_one_launch_normalises(B):
    import torch
    per = (2**32 - 1) // 64                                   # a workgroup of 64 threads a row
    rows, cols = per + 300, 8
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV).normal_()
    w = torch.full((cols,), 1.5, dtype=torch.bfloat16, device=DEV)
    codes, scales = torch.full((rows, cols), 99, dtype=torch.int8, device=DEV), torch.full((rows,), -1.0, device=DEV)
    B.add_rms_norm(x, w, codes, 1e-5, scales=scales)
    torch.cuda.synchronize()
    assert bool((scales > 0).all())
    for at in (slice(0, 50), slice(2**26 - 30, 2**26 + 30), slice(per - 50, per + 50), slice(rows - 50, rows)):
        y, _ = L.rms_norm_rows(x[at].float().cpu().numpy(), None, np.full(cols, 1.5, np.float32), 1e-5)
        c, s = L.int8_rows(y)
        assert np.array_equal(codes[at].cpu().numpy(), c) and np.array_equal(scales[at].cpu().numpy(), s)


def test_more_rows_than_one_launch_turns(B):
    import torch
    per = (2**32 - 1) // 256 * 4                              # a wavefront a row
    rows = per + 300
    q = torch.empty((rows, 1, 16), dtype=torch.bfloat16, device=DEV).normal_()
    spots = [slice(0, 40), slice(2**26 - 30, 2**26 + 30), slice(per - 40, per + 40), slice(rows - 40, rows)]
    before = [q[at].float().cpu().numpy() for at in spots]
    pos = torch.arange(rows, dtype=torch.int32, device=DEV)
    f, _ = B.rotary_frequencies(16)
    B.rotary(q, None, pos, f.to(DEV))
    torch.cuda.synchronize()
    for at, x in zip(spots, before):
        want = L.rotary(x, np.arange(at.start, at.stop), f.numpy())
        size = np.abs(x) + np.abs(np.roll(x, 8, -1))
        assert (np.abs(q[at].float().cpu().numpy() - want) <= 5e-7 * size + 2.0 ** -8 * np.abs(want) + 1e-38).all()


@pytest.mark.parametrize("cache", ["same", "blocks"])
def test_blocks_behind_4_gib(B, cache):
    import torch
    from test_gpu_decode_shared import Case
    case = Case([(400, [405 + i for i in range(13)]), (100, [120, 130])], [77], cache=cache, seed=51)
    small = case.device()
    per = small["cache"][0].numel() * small["cache"].element_size()
    blocks = (5 << 30) // per
    big, shift = dict(small), blocks - case.num_blocks
    big["cache"] = torch.empty((blocks,) + tuple(small["cache"].shape[1:]), dtype=small["cache"].dtype, device=DEV)
    big["cache"][shift:] = small["cache"]
    if cache == "blocks":
        big["scales"] = torch.ones((blocks, 1, 2), device=DEV)
        big["scales"][shift:] = small["scales"]
    big["table"] = torch.where(small["table"] >= 0, small["table"] + shift, small["table"])
    big["slots"] = small["slots"] + 16 * shift
    big["out"] = torch.zeros_like(small["out"])
    try:
        B.set_option(B.OPT_DECODE_SHARED, 1)
        case.call(B, big)
        case.call(B, small)
    finally:
        B.set_option(B.OPT_DECODE_SHARED, 0)
    torch.cuda.synchronize()
    case.check(small)
    assert torch.equal(big["out"], small["out"]) and torch.equal(big["cache"][shift:].view(torch.uint8), small["cache"].view(torch.uint8))
