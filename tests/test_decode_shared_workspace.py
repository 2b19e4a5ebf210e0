"""decode_shared_workspace_bytes holds every smaller call (host only): a server that asks once for its largest batch is never refused later."""
import random

import pytest

from test_layer_refusals import B, _attn


@pytest.mark.parametrize("option", [0, 1, 2])
def test_no_smaller_call_needs_more(B, option):
    rng = random.Random(option)
    log = lambda lo, hi: min(hi, max(lo, int(lo * (hi / lo) ** rng.random())))
    try:
        B.set_option(B.OPT_DECODE_SHARED, option)
        for _ in range(4000):
            hkv, G = rng.choice([(1, 8), (8, 4), (1, 16), (3, 1), (64, 2)])
            a = _attn(B, num_kv_heads=hkv, num_q_heads=hkv * G, max_blocks_per_seq=1 << 27)
            most = [log(1, 4000), log(1, 2**31 - 65), 0]
            most[2] = rng.randint(0, max(most[0], 512))
            less = [rng.choice([n, log(1, n), max(1, n - 1)]) for n in most[:2]]
            less.append(rng.choice([most[2], rng.randint(0, most[2]), min(most[2], 512), min(most[2], 513)]))
            size = B.decode_shared_workspace_bytes(*most, a)
            assert size >= B.decode_shared_workspace_bytes(*less, a), (most, less, hkv, G)
            assert size >= B.decode_workspace_bytes(less[0], less[1], a), (most, less, hkv, G)
    finally:
        B.set_option(B.OPT_DECODE_SHARED, 0)


def test_on_both_sides_of_what_is_indexed(B):
    """600 groups take the plain kernel, 300 of the same server's next batch the one that shares; 2^23 tokens make launches of fewer sequences than 2^20."""
    a = _attn(B, max_blocks_per_seq=1 << 20)
    assert B.decode_shared_workspace_bytes(1200, 4000, 600, a) >= B.decode_shared_workspace_bytes(1200, 4000, 300, a) > B.decode_workspace_bytes(1200, 4000, a)
    assert B.decode_shared_workspace_bytes(1024, 2**23, 512, a) >= B.decode_shared_workspace_bytes(1024, 2**20, 512, a)
