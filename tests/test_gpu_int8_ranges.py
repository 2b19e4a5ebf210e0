"""int8 products whose rows end in half a stage (k an odd multiple of 64) and whose k is split over workgroups: the range that holds the
last stage leaves out what lies behind the row, and the ranges' integers add up to the same bits."""
import numpy as np
import pytest

from test_gpu_int8 import _codes, _dev, _product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,h,h_kv,K", [(3, 4, 2, 8256), (48, 4, 2, 4160), (140, 4, 2, 4160), (140, 4, 2, 16448), (520, 4, 2, 4160), (900, 14, 2, 16448)])
def test_k_ranges_that_end_in_half_a_stage(T, h, h_kv, K):
    import torch
    from paper_2509_16495_amd import binding as B
    N = (h + 2 * h_kv) * 128
    plan = B.proj_plan(T, N, K, fp8=True)
    assert plan.k_ranges > 1 and not plan.streams
    rng = np.random.Generator(np.random.PCG64(K + T))
    xc, xs = _codes(rng, T, K)
    wc, ws = _codes(rng, N, K)
    send = torch.full((2, T, (h + 2 * h_kv) // 2, 128), np.nan, dtype=torch.bfloat16, device="cuda")
    work = torch.full((B.proj_workspace_bytes_int8(T, N, K),), 0xA5, dtype=torch.uint8, device="cuda")
    B.qkv_proj_pack_int8(_dev(xc), _dev(xs), _dev(wc), _dev(ws), send, 2, h, h_kv, workspace=work)
    y = _product(xc, xs, wc, ws).reshape(T, h + 2 * h_kv, 128)
    heads = [np.r_[p * h // 2:(p + 1) * h // 2, h + p * h_kv // 2:h + (p + 1) * h_kv // 2, h + h_kv + p * h_kv // 2:h + h_kv + (p + 1) * h_kv // 2] for p in (0, 1)]
    got, want = send.float().cpu().numpy(), np.stack([y[:, i] for i in heads])
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]
