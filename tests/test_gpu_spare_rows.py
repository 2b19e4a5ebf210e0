"""Rows that stand for no token: a batch with fewer tokens than the host set rows aside for, as when block tables built on the GPU refuse a
chunk.  Every kernel leaves their rows of the result as they were and gives the other rows what they get without them."""
import contextlib

import numpy as np
import pytest

import plain_8bit as P

pytestmark = pytest.mark.gpu

MARK = 7.0   # what the result holds before the call


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    binding.lib()
    return binding


@contextlib.contextmanager
def _option(B, name, value):
    if name:
        B.set_option(getattr(B, name), value)
    try:
        yield
    finally:
        if name:
            B.set_option(getattr(B, name), 0)


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.to(torch.bfloat16).cuda() if dtype == "bf16" else t.cuda()


def _rows(rng, *shape, dtype):
    x = rng.standard_normal(shape).astype(np.float32)
    return P.bf16(x) if dtype == "bf16" else x


class Values:
    """A cache of values as they are, in the place of P.Cache."""

    def __init__(self, num_blocks, heads, D):
        self.heads, self.x = heads, np.zeros((num_blocks, heads, 2, 16, D), np.float32)

    def append(self, k, v, slots):
        for i, slot in enumerate(slots):
            if slot >= 0:
                self.x[slot // 16, :, 0, slot % 16], self.x[slot // 16, :, 1, slot % 16] = k[i], v[i]

    def rows(self, table, length, g, part):
        return np.concatenate([self.x[b, g, part] for b in table[:-(-length // 16)]])[:length].astype(np.float64)

    def device(self, dtype):
        a = self.x.copy()
        n, h, _, _, D = a.shape
        a[:, :, 1] = a[:, :, 1].swapaxes(2, 3).reshape(n, h, 16, D)   # (the bytes of V [D][16])
        return _dev(a.reshape(n, h, 2, 16 * D), dtype)


class Step:
    """Tables whose blocks run out, built on the GPU: chunks of which some are refused, `spare` rows more than the chunks ask for, decode rows."""

    def __init__(self, B, fmt, dtype, D, hq, hkv, had, new, blocks_left, spare, decs, seed):
        import torch
        rng = np.random.Generator(np.random.PCG64(seed))
        seqs, n_pre = len(had) + len(decs), len(had)
        lens = list(had) + [c - 1 for c in decs]
        used = [-(-n // 16) for n in lens]
        wide = max(-(-(n + m) // 16) for n, m in zip(lens, list(new) + [1] * len(decs)))
        num_blocks = sum(used) + blocks_left
        ids = rng.permutation(num_blocks).astype(np.int32)
        plain = P.Tables(lens, wide, np.r_[ids[sum(used):], np.zeros(sum(used), np.int32)], num_blocks - sum(used))
        at = 0
        for s, n in enumerate(used):
            plain.table[s, :n] = ids[at:at + n]
            at += n
        self.cache = P.Cache(num_blocks, hkv, D, rng) if fmt == "scaled" else Values(num_blocks, hkv, D)
        for s, n in enumerate(lens):
            x = _rows(rng, n, hkv, 2 * D, dtype=dtype)
            self.cache.append(x[..., :D], x[..., D:], plain.table[s, np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16)
        self.kv = dict(kv_scales=_dev(self.cache.scales)) if fmt == "scaled" else {}
        codes = _dev(self.cache.codes) if fmt == "scaled" else self.cache.device(dtype)
        total = sum(new) + spare
        rows = total + len(decs)
        new_all = np.array(list(new) + [1] * len(decs), np.int32)
        dev = [_dev(np.asarray(x, np.int32)) for x in (plain.lens, plain.table, plain.free, [plain.count])]
        cu, slots = torch.empty(n_pre + 1, dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.int64, device="cuda")
        taken = torch.empty(seqs, dtype=torch.int32, device="cuda")
        B.tables_append(_dev(new_all), n_pre, total, *dev, cu, slots, taken)
        want_cu, want_slots, want_taken = plain.append(new_all, n_pre, total, rows)
        assert np.array_equal(cu.cpu().numpy(), want_cu) and np.array_equal(slots.cpu().numpy(), want_slots) and np.array_equal(taken.cpu().numpy(), want_taken)
        self.tokens = int(want_cu[-1])
        assert self.tokens < total
        q, k, v = (_rows(rng, rows, h, D, dtype=dtype) for h in (hq, hkv, hkv))
        q[self.tokens:total] = k[self.tokens:total] = v[self.tokens:total] = np.nan    # nothing of these rows may reach the others
        self.cache.append(k, v, want_slots)
        self.plain, self.total, self.q, self.codes, self.lens, self.table, self.cu = plain, total, q, codes, dev[0], dev[1], cu
        self.dtype, self.D, self.n_pre, self.decs, self.new, self.taken = dtype, D, n_pre, decs, new, want_taken
        self.dev_q, self.out = _dev(q, dtype), torch.full((rows, hq, D), MARK, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
        self.append = dict(k_new=_dev(k, dtype), v_new=_dev(v, dtype), slot_mapping=slots)
        self.longest = wide * 16

    def check(self):
        got = self.out.float().cpu().numpy().astype(np.float64)
        total, cu = self.total, self.cu.cpu().numpy()
        assert (got[self.tokens:total] == MARK).all()
        spans = [(int(cu[s]), int(cu[s + 1]), s) for s in range(self.n_pre)] + [(total + j, total + j + 1, self.n_pre + j) for j in range(len(self.decs))]
        for lo, hi, s in spans:
            n = int(self.plain.lens[s])
            if hi > lo and n > 0:
                want = P.attend(self.q[lo:hi], self.cache, self.plain.table[s], n, self.D ** -0.5)
                off = np.abs(got[lo:hi] - want[0]) / P.bound(self.dtype, *want, self.D, n)
                assert off.max() <= 1.0, (s, off.max())


KINDS = [("scaled", "bf16", 128, 8, 1), ("scaled", "bf16", 64, 4, 1), ("scaled", "f32", 64, 4, 2), ("scaled", "bf16", 256, 2, 1), ("same", "bf16", 128, 8, 1),
         ("same", "bf16", 64, 4, 1), ("same", "f32", 64, 4, 1), ("same", "f32", 80, 2, 1)]
# chunks on cached tokens, their new tokens, blocks that are left for them, rows more than asked for: a refused chunk behind, between and in front
# of others, all of them, none (rows to spare only)
BATCHES = [([5, 20], [4, 40], 0, 0), ([5, 200, 40], [30, 90, 8], 2, 3), ([33, 3], [100, 5], 1, 0), ([16, 32], [20, 50], 0, 0), ([0, 70], [21, 130], 20, 37)]


@pytest.mark.parametrize("option,value", [(None, 0), ("OPT_GENERIC_ONLY", 1), ("OPT_PREFILL_SPLITS", 3)])
@pytest.mark.parametrize("fmt,dtype,D,hq,hkv", KINDS)
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_prefill(B, fmt, dtype, D, hq, hkv, batch, option, value):
    had, new, left, spare = BATCHES[batch]
    st = Step(B, fmt, dtype, D, hq, hkv, had, new, left, spare, [], batch)
    with _option(B, option, value):
        B.prefill(st.dev_q, st.codes, st.table, st.cu, st.lens, max(new), st.longest, st.out, D ** -0.5, **st.append, **st.kv)
    st.check()


@pytest.mark.parametrize("option,value", [(None, 0), ("OPT_GENERIC_ONLY", 1), ("OPT_PREFILL_SPLITS", 3)])
@pytest.mark.parametrize("fmt,dtype,D,hq,hkv", KINDS)
@pytest.mark.parametrize("batch", range(len(BATCHES)))
def test_mixed(B, fmt, dtype, D, hq, hkv, batch, option, value):
    had, new, left, spare = BATCHES[batch]
    st = Step(B, fmt, dtype, D, hq, hkv, had, new, left, spare, [1, 30, 17, 150], 10 + batch)
    with _option(B, option, value):
        B.mixed(st.dev_q, st.codes, st.table, st.cu, st.lens, len(had), max(new), st.longest, st.longest, st.out, D ** -0.5, **st.append, **st.kv)
    st.check()


@pytest.mark.parametrize("fmt", ["scaled", "same"])
def test_chunks_and_rows_in_one_launch(B, fmt):
    """A unified batch whose decode rows go into the prefill kernel's launch, its key ranges merged with them."""
    st = Step(B, fmt, "bf16", 128, 8, 1, [2000, 900], [300, 200], 19, 11, [40 + 30 * i for i in range(60)], 30)
    a = B.attn_desc(st.dev_q, st.codes, st.table, 128 ** -0.5, None, st.out, **st.kv)
    plan = B.prefill_plan(2, st.total, 300, st.longest, a, 60, 1810)
    assert plan.decode_wgs > 0 and plan.key_ranges > 1, (plan.decode_wgs, plan.key_ranges)
    B.mixed(st.dev_q, st.codes, st.table, st.cu, st.lens, 2, 300, st.longest, 1810, st.out, 128 ** -0.5, **st.append, **st.kv)
    st.check()
