"""Lengths that the tables' rows cannot hold: neither call follows them behind a row."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


@pytest.mark.parametrize("seqs,num_blocks", [(6, 40), (1030, 4200), (6, 70000)])   # one launch, more sequences than one holds, more blocks than one gives back
def test_truncate_leaves_lengths_beyond_their_row(B, seqs, num_blocks):
    """Rows of three blocks; every third sequence says that it has more tokens than 48."""
    import torch
    wide = 3 if num_blocks < 70000 else 20000
    row = wide * 16
    lens = np.array([[row + 1, 33, row], [2 ** 31 - 1, 16, row + 16]] * (seqs // 6 + 1), np.int64).reshape(-1)[:seqs]
    table = np.arange(1, 1 + seqs * wide).reshape(seqs, wide)
    keep = np.array([0, 17, row - 16, 1, 0, row] * (seqs // 6 + 1))[:seqs]
    dev = [_dev(x) for x in (lens, table, np.full(num_blocks, -3), [5])]
    B.tables_truncate(_dev(keep), *dev)
    back, want_lens = [], lens.copy()
    for s in range(seqs):
        if lens[s] <= row and keep[s] < lens[s]:
            back += table[s, -(-keep[s] // 16):-(-lens[s] // 16)].tolist()
            want_lens[s] = keep[s]
    free = np.full(num_blocks, -3)
    free[5:5 + len(back)] = back[::-1]
    assert np.array_equal(dev[0].cpu().numpy(), want_lens) and int(dev[3]) == 5 + len(back)
    assert np.array_equal(dev[2].cpu().numpy(), free) and np.array_equal(dev[1].cpu().numpy(), table)
    # and an append refuses them, as before
    cu, slots, taken = _dev([0]), torch.empty(seqs, dtype=torch.int64, device="cuda"), _dev(np.zeros(seqs))
    B.tables_append(_dev(np.ones(seqs)), 0, 0, *dev, cu, slots, taken)
    assert not taken.cpu().numpy()[want_lens > row].any() and (slots.cpu().numpy()[want_lens > row] == -1).all()
