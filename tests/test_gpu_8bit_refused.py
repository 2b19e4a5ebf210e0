"""Steps of an engine that serves in 8 bits whose blocks run out: tables built on the GPU refuse chunks and decode rows, rows are set aside that
nobody asked for, and every operator behind them takes what is there, with the counts that the host passed."""
import numpy as np
import pytest

import plain_8bit as P
from test_gpu_8bit_step import D_MODEL, Engine, _dev, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


# new tokens, chunks among them, rows to spare, tokens kept behind the step
SCRIPTS = {
    "behind others": (9, [([40, 70, 20, 33, 16], 5, 0, None), ([5, 60, 1, 1, 1], 2, 3, None), ([1, 1, 1, 1, 1], 0, 0, [0, -1, -1, -1, -1]), ([30, 40, 1, 0, 1], 2, 0, None)]),
    "in front of others": (6, [([100, 10, 20], 3, 2, None), ([16, 5, 1], 2, 0, None), ([90, 2, 1], 2, 7, [-1, 0, 0]), ([70, 9, 1], 2, 0, None)]),
    "all": (3, [([90, 64], 2, 0, None), ([33, 1], 1, 5, None), ([200, 1], 1, 0, None)]),
}


@pytest.mark.parametrize("name", SCRIPTS)
def test_steps_with_refused_chunks(B, name):
    import torch
    rng = np.random.Generator(np.random.PCG64(31))
    blocks, script = SCRIPTS[name]
    e, refused = Engine(B, len(script[0][0]), 16, blocks, rng), 0
    for new, n_pre, spare, keep in script:
        total = sum(new[:n_pre]) + spare
        rows = total + len(new) - n_pre
        e.buffers(rows, n_pre)
        e.attn.fill_(0.5)
        x = P.bf16(rng.standard_normal((rows, D_MODEL)).astype(np.float32) * np.exp(rng.standard_normal((rows, 1))).astype(np.float32))
        e.x.copy_(_dev(x).to(torch.bfloat16))
        e.step(_dev(np.array(new, np.int32)), n_pre, total, max(new[:n_pre], default=0), 16 * 16)
        e.check(x, new, n_pre, total)
        there = int(e.cu[-1])
        assert (_np(e.attn[0])[there:total] == 0.5).all()
        refused += total - there
        if keep:
            e.truncate(keep)
    assert refused > 0
