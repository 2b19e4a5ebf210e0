"""Block tables and slot maps built on the GPU against the sequential implementation: whole numbers, equal."""
import numpy as np
import pytest

import plain_8bit as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


def _dev(a, dtype=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


class OnGpu:
    """The same state on the GPU."""

    def __init__(self, B, plain, num_prefill):
        import torch
        self.B, self.n_pre, n = B, num_prefill, len(plain.lens)
        self.lens, self.table, self.free, self.count = _dev(plain.lens), _dev(plain.table), _dev(plain.free), _dev([plain.count])
        self.cu, self.taken = torch.full((num_prefill + 1,), -7, dtype=torch.int32, device="cuda"), torch.full((n,), -7, dtype=torch.int32, device="cuda")
        self.ws = torch.full((B.tables_workspace_bytes(n),), 0xA5, dtype=torch.uint8, device="cuda")

    def append(self, new, total, rows):
        import torch
        self.slots = torch.full((rows,), -9, dtype=torch.int64, device="cuda")
        self.B.tables_append(_dev(new), self.n_pre, total, self.lens, self.table, self.free, self.count, self.cu, self.slots, self.taken, self.ws)

    def truncate(self, keep):
        self.B.tables_truncate(_dev(keep), self.lens, self.table, self.free, self.count, self.ws)

    def same(self, plain, result=None):
        assert np.array_equal(self.lens.cpu().numpy(), plain.lens) and int(self.count) == plain.count
        assert np.array_equal(self.table.cpu().numpy(), plain.table) and np.array_equal(self.free.cpu().numpy(), plain.free)
        if result is not None:
            for got, want in zip((self.cu, self.slots, self.taken), result):
                assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("seqs,n_pre,longest,blocks", [
    (1, 0, 1, 3), (1, 1, 1, 1), (1, 1, 5000, 400), (5, 5, 40, 60), (61, 0, 1, 700), (285, 29, 3000, 9000), (1024, 0, 1, 3000), (1025, 1025, 20, 4000),
    (2500, 700, 90, 9000), (3, 2, 70000, 9000), (64, 32, 40, 10), (9, 4, 30, 0)])
def test_steps_of_an_engine(B, seqs, n_pre, longest, blocks):
    """Steps of random lengths: some sequences idle, some of them cut back or finished between the steps, blocks and rows now and then too
    few."""
    rng = np.random.Generator(np.random.PCG64(seqs * 7 + n_pre))
    plain = P.Tables(rng.integers(-2, 1, seqs), max(1, 2 * longest // 16 + 3), rng.permutation(blocks), blocks)
    gpu = OnGpu(B, plain, n_pre)
    for step in range(6):
        new = np.where(np.arange(seqs) < n_pre, rng.integers(-1, longest + 1, seqs), rng.integers(0, 3 if step == 4 else 2, seqs))
        asked = int(np.maximum(new[:n_pre], 0).sum())
        total = [asked, asked + 5, asked // 2][step % 3]
        rows = total + seqs - n_pre + [0, 3][step % 2]
        result = plain.append(new, n_pre, total, rows)
        gpu.append(new, total, rows)
        gpu.same(plain, result)
        keep = np.where(rng.random(seqs) < 0.5, -1, (np.maximum(plain.lens, 0) * rng.random(seqs) * 1.2).astype(int))
        keep[rng.random(seqs) < 0.2] = 0
        plain.truncate(keep)
        gpu.truncate(keep)
        gpu.same(plain)


def test_a_truncate_undoes_an_append(B):
    rng = np.random.Generator(np.random.PCG64(8))
    plain = P.Tables([0] * 50, 100, rng.permutation(2000), 2000)
    gpu = OnGpu(B, plain, 20)
    gpu.append(np.r_[rng.integers(0, 900, 20), np.ones(30, int)], 18000, 18032)
    before = gpu.lens.cpu().numpy(), gpu.free.cpu().numpy(), int(gpu.count)
    gpu.append(np.r_[rng.integers(0, 300, 20), np.ones(30, int)], 6000, 6030)
    assert int(gpu.count) < before[2] and int(gpu.taken.sum()) > 30
    gpu.truncate(before[0])
    assert np.array_equal(gpu.lens.cpu().numpy(), before[0]) and np.array_equal(gpu.free.cpu().numpy(), before[1]) and int(gpu.count) == before[2]


def test_counts_outside_the_stack_are_taken_as_its_ends(B):
    for count in (-5, 99):
        plain = P.Tables([0, 0], 4, np.arange(6), count)
        gpu = OnGpu(B, plain, 0)
        result = plain.append([1, 1], 0, 0, 2)
        gpu.append([1, 1], 0, 2)
        gpu.same(plain, result)


def test_lengths_near_the_end_of_32_bits(B):
    """Sums of what is asked for beyond 2^31: refused, nothing wraps."""
    plain = P.Tables([0, 5, 0, 2 ** 31 - 20, 0], 3, np.arange(9), 9)
    gpu = OnGpu(B, plain, 5)
    new = [40, 2 ** 31 - 1, 2 ** 31 - 1, 30, 2]
    result = plain.append(new, 5, 50, 50)
    gpu.append(new, 50, 50)
    gpu.same(plain, result)
    assert result[2].tolist() == [40, 0, 0, 0, 2]


def test_lengths_stay_below_2_31(B):
    """A row of block_table that could hold more tokens than an int32 length can say."""
    import torch
    wide = 2 ** 27 + 2
    table, lens, free = torch.zeros((1, wide), dtype=torch.int32, device="cuda"), _dev([2 ** 31 - 20]), _dev([5, 6, 7])
    count, cu, slots, taken = _dev([3]), _dev([0, 0]), _dev(np.zeros(40), np.int64), _dev([0])
    for new, want in ((30, 0), (20, 0), (19, 19)):
        B.tables_append(_dev([new]), 1, 40, lens, table, free, count, cu, slots, taken)
        assert taken.tolist() == [want] and cu.tolist() == [0, want] and lens.tolist() == [2 ** 31 - 20 + want] and int((slots >= 0).sum()) == want
    # offsets 12 .. 15 of the block that was there (0), then those of the block taken
    assert count.tolist() == [2] and int(table[0, 2 ** 27 - 1]) == 7 and slots[:19].tolist() == [12, 13, 14, 15] + list(range(112, 127))


def test_no_sequences_leave_an_empty_map(B):
    import torch
    plain = P.Tables([], 4, np.arange(3), 3)
    gpu = OnGpu(B, plain, 0)
    gpu.append([], 0, 5)
    gpu.truncate([])
    assert gpu.cu.tolist() == [0] and gpu.slots.tolist() == [-1] * 5 and int(gpu.count) == 3
    torch.cuda.synchronize()


def test_replayed_from_a_graph_on_a_stream_of_its_own(B):
    """A decode step's append, captured once: the state moves on in device memory from replay to replay."""
    import torch
    rng = np.random.Generator(np.random.PCG64(9))
    plain = P.Tables(rng.integers(0, 60, 37), 8, rng.permutation(300), 300)
    for s in range(37):   # blocks of the tokens that are there
        for b in range(-(-int(plain.lens[s]) // 16)):
            plain.count -= 1
            plain.table[s, b] = plain.free[plain.count]
    gpu, new = OnGpu(B, plain, 0), torch.ones(37, dtype=torch.int32, device="cuda")
    gpu.slots = torch.zeros(40, dtype=torch.int64, device="cuda")
    start = [t.clone() for t in (gpu.lens, gpu.table, gpu.free, gpu.count)]
    st = torch.cuda.Stream()
    call = lambda: B.tables_append(new, 0, 0, gpu.lens, gpu.table, gpu.free, gpu.count, gpu.cu, gpu.slots, gpu.taken, gpu.ws)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        call()
    torch.cuda.current_stream().wait_stream(st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t, v in zip((gpu.lens, gpu.table, gpu.free, gpu.count), start):
        t.copy_(v)
    for step in range(90):
        graph.replay()
        if step % 3 == 0:   # the program's own work between replays
            torch.cuda.synchronize()
            gpu.slots.add_(0)
        result = plain.append([1] * 37, 0, 0, 40)
        gpu.same(plain, result)
    assert 0 in result[2].tolist()   # sequences that reached the end of their rows
