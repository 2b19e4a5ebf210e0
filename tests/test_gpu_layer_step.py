"""Decode steps of a layer for a batch behind one prompt, from the residual stream to the residual stream: blocks and slots on the GPU, residual
addition and norm into int8, q|k|v projection, rotary positions on the rows it left, attention over the cache with block scales whose
first blocks all sequences share (with its append), output projection, the next norm.  Every stage is held to the plain implementation on what
the stage in front of it left, so that the bounds are those of one stage."""
import numpy as np
import pytest

import plain_8bit as P
import plain_layer as L

pytestmark = pytest.mark.gpu

D, H, H_KV, D_MODEL, EPS = 128, 8, 2, 512, 1e-5
PROMPT, MAX_BLOCKS = 168, 16          # ten whole blocks in common; the prompt's last eight tokens are each sequence's own


@pytest.fixture(scope="module")
def B():
    """The kernel that shares takes these batches too, which are the plain kernel's by their size."""
    from paper_2509_16495_amd import binding
    binding.lib()
    binding.set_option(binding.OPT_DECODE_SHARED, 1)
    yield binding
    binding.set_option(binding.OPT_DECODE_SHARED, 0)


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _np(t):
    return t.float().cpu().numpy()


class Layer:
    """`seqs` sequences whose caches hold the prompt, the first 10 blocks of it once for all."""

    def __init__(self, B, seqs, rng, residual_bf16=True):
        import torch
        self.B, self.seqs, self.rng, self.res_bf16 = B, seqs, rng, residual_bf16
        self.wq, self.wqs = P.quantise_int8(P.bf16(rng.standard_normal(((H + 2 * H_KV) * D, D_MODEL)).astype(np.float32) * np.float32(D_MODEL ** -0.5)))
        self.wo, self.wos = P.quantise_int8(P.bf16(rng.standard_normal((D_MODEL, H * D)).astype(np.float32) * np.float32((H * D) ** -0.5)))
        self.w1, self.w2 = (P.bf16(1 + 0.2 * rng.standard_normal(D_MODEL).astype(np.float32)) for _ in range(2))
        common = PROMPT // 16
        num_blocks = common + seqs * (MAX_BLOCKS - common)
        order = rng.permutation(num_blocks).astype(np.int32)
        self.cache = P.Cache(num_blocks, H_KV, D, rng)
        self.table = rng.integers(0, num_blocks, (seqs, MAX_BLOCKS)).astype(np.int32)
        self.table[:, :common] = order[:common]
        self.table[:, common] = order[common:common + seqs]
        for s in range(seqs):
            for blk in np.concatenate([self.table[0, :common] if s == 0 else [], self.table[s, common:common + 1]]).astype(int):
                k, v = (rng.standard_normal((16, H_KV, D)).astype(np.float32) for _ in range(2))
                self.cache.append(k, v, blk * 16 + np.arange(16))
        self.free, self.used = order[common + seqs:][::-1].copy(), num_blocks - common - seqs
        self.lens = np.full(seqs, PROMPT, np.int64)
        i = lambda a: _dev(np.asarray(a, np.int32))
        e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
        self.d = d = {}
        d["table"], d["lens"], d["count"] = i(self.table), i(self.lens), i([self.used])
        d["free"] = i(np.concatenate([self.free, np.zeros(num_blocks - self.used)]))
        d["codes"], d["scales"] = _dev(self.cache.codes), _dev(self.cache.scales)
        d["new"], d["taken"], d["cu"], d["slots"] = i(np.zeros(seqs)), i(np.zeros(seqs)), i([0]), e(seqs, dtype=torch.int64)
        d["groups"], d["shared"] = i([0, seqs]), i([PROMPT])
        d["x"], d["stream"], d["xc"], d["xs"] = e(seqs, D_MODEL), e(seqs, D_MODEL, dtype=torch.bfloat16 if residual_bf16 else torch.float32), e(seqs, D_MODEL, dtype=torch.int8), e(seqs, dtype=torch.float32)
        d["send"], d["attn"], d["ac"], d["as"] = e(1, seqs, H + 2 * H_KV, D), e(1, seqs, H, D), e(1, seqs, H, D, dtype=torch.int8), e(seqs, dtype=torch.float32)
        d["y"], d["next"] = e(seqs, D_MODEL), e(seqs, D_MODEL)
        d["w1"], d["w2"] = (_dev(w).to(torch.bfloat16) for w in (self.w1, self.w2))
        d["wq"], d["wqs"], d["wo"], d["wos"] = (_dev(w) for w in (self.wq, self.wqs, self.wo, self.wos))
        self.freq, _ = B.rotary_frequencies(D, 10000.0, "wavelengths", 8.0, 128.0, 1.0, 4.0)
        d["freq"] = self.freq.cuda()
        self.qkv = None

    def step(self, watch=lambda: None):
        B, d = self.B, self.d
        rows = d["send"][0]
        B.tables_append(d["new"], 0, 0, d["lens"], d["table"], d["free"], d["count"], d["cu"], d["slots"], d["taken"])
        B.add_rms_norm(d["x"], d["w1"], d["xc"], EPS, residual=d["stream"], scales=d["xs"])
        B.qkv_proj_pack_int8(d["xc"], d["xs"], d["wq"], d["wqs"], d["send"], 1, H, H_KV)
        watch()
        B.rotary_mixed(rows[:, :H], rows[:, H:H + H_KV], d["cu"], d["lens"], 0, d["freq"])
        B.decode_shared(rows[:, :H], d["codes"], d["table"], d["lens"], MAX_BLOCKS * 16, d["groups"], d["shared"], d["attn"][0], D ** -0.5,
                        k_new=rows[:, H:H + H_KV], v_new=rows[:, H + H_KV:], slot_mapping=d["slots"], kv_scales=d["scales"])
        B.quantize_recv_int8(d["attn"], d["ac"], d["as"])
        B.unpack_o_proj_int8(d["ac"], d["as"], d["wo"], d["wos"], d["y"])
        B.add_rms_norm(d["y"], d["w2"], d["next"], EPS, residual=d["stream"])

    def feed(self, new):
        """Inputs of the next step."""
        import torch
        self.new = np.asarray(new)
        self.x = P.bf16(self.rng.standard_normal((self.seqs, D_MODEL)).astype(np.float32) * np.exp(self.rng.standard_normal((self.seqs, 1))).astype(np.float32))
        s = self.rng.standard_normal((self.seqs, D_MODEL)).astype(np.float32) * 3
        self.stream = P.bf16(s) if self.res_bf16 else s
        self.d["new"].copy_(_dev(self.new.astype(np.int32)))
        self.d["x"].copy_(_dev(self.x))
        self.d["stream"].copy_(_dev(self.stream))
        torch.cuda.synchronize()

    def check(self):
        d = self.d
        # blocks from the top of the stack, in the order of sequences
        slots = np.full(self.seqs, -1)
        for s in range(self.seqs):
            if self.new[s]:
                p = self.lens[s]
                if p % 16 == 0:
                    self.used -= 1
                    self.table[s, p // 16] = self.free[self.used]
                slots[s] = self.table[s, p // 16] * 16 + p % 16
                self.lens[s] += 1
        assert np.array_equal(d["slots"].cpu().numpy(), slots) and np.array_equal(d["lens"].cpu().numpy(), self.lens)
        y, stream = L.rms_norm_rows(self.x, self.stream, self.w1, EPS, residual_bf16=self.res_bf16)
        c, sc = L.int8_rows(y)
        assert np.array_equal(d["xc"].cpu().numpy(), c) and np.array_equal(d["xs"].cpu().numpy(), sc)
        product = lambda c, s, w, ws: P.bf16((c.astype(np.float64) @ w.T.astype(np.float64)).astype(np.float32) * s[:, None] * ws)
        qkv = product(c, sc, self.wq, self.wqs).reshape(self.seqs, H + 2 * H_KV, D)
        rows = _np(d["send"][0])
        want = L.rotary(qkv[:, :H + H_KV], self.lens - 1, self.freq.numpy())
        size = np.abs(qkv[:, :H + H_KV])
        bound = 5e-7 * (size + np.roll(size, D // 2, -1)) + 2.0 ** -8 * np.abs(want) + 1e-38
        assert (np.abs(rows[:, :H + H_KV] - want) <= bound).all() and np.array_equal(rows[:, H + H_KV:], qkv[:, H + H_KV:])
        self.cache.append(rows[:, H:H + H_KV], rows[:, H + H_KV:], slots)
        assert np.array_equal(d["codes"].cpu().numpy(), self.cache.codes) and np.array_equal(d["scales"].cpu().numpy(), self.cache.scales)
        attn = _np(d["attn"][0])
        for s in range(self.seqs):
            want = P.attend(rows[s:s + 1, :H], self.cache, self.table[s], int(self.lens[s]), D ** -0.5)
            off = np.abs(attn[s:s + 1] - want[0]) / P.bound("bf16", *want, D, int(self.lens[s]))
            assert off.max() <= 1.0, (s, off.max())
        c, sc = P.quantise_int8(attn.reshape(self.seqs, H * D))
        assert np.array_equal(_np(d["y"]), product(c, sc, self.wo, self.wos))
        y, stream = L.rms_norm_rows(_np(d["y"]), stream, self.w2, EPS, residual_bf16=self.res_bf16)
        assert np.array_equal(_np(d["stream"]), stream) and np.array_equal(_np(d["next"]), P.bf16(y))


@pytest.mark.parametrize("seqs,residual_bf16", [(2, True), (7, False), (21, True)])
def test_steps(B, seqs, residual_bf16):
    rng = np.random.Generator(np.random.PCG64(seqs))
    layer = Layer(B, seqs, rng, residual_bf16)
    for step in range(12):
        layer.feed([1] * seqs if step % 3 else rng.integers(0, 2, seqs))     # (a sequence without a token attends to what it has)
        layer.step()
        layer.check()
    assert layer.lens.max() > 176          # (into blocks that the steps took)


def test_steps_from_one_graph_on_a_stream_of_its_own(B):
    import torch
    rng = np.random.Generator(np.random.PCG64(5))
    layer = Layer(B, 9, rng)
    side = torch.cuda.Stream()
    layer.feed([0] * 9)
    with torch.cuda.stream(side):
        layer.step()                             # no new tokens: nothing moves but the stream
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.step()
    for step in range(20):
        layer.feed([1] * 9)
        graph.replay()
        if step % 3 == 0:
            _ = (layer.d["y"].float() * 2).sum().item()
        layer.check()


def test_two_graphs_that_share_a_workspace(B):
    """Calls of one stream may share a workspace, captured or not: what one leaves there is nothing to the next."""
    import torch
    from test_gpu_decode_shared import Case
    cases = [Case([(300, [310 + i for i in range(11)])], [90], seed=1), Case([(64, [70, 77]), (500, [505, 620, 700])], cache="blocks", seed=2)]
    ds = [c.device() for c in cases]
    sizes = []
    for c, d in zip(cases, ds):
        a = B.attn_desc(d["q"], d["cache"], d["table"], c.scale, d["k"], d["out"], *c.factors, d["scales"])
        sizes.append(B.decode_shared_workspace_bytes(len(c.lens), int(c.lens.max()), len(c.shared_lens), a))
    ws = torch.full((max(sizes),), 0xFF, dtype=torch.uint8, device="cuda")
    graphs = []
    for c, d in zip(cases, ds):
        c.call(B, d, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.call(B, d, workspace=ws)
        graphs.append(g)
    for i in (0, 1, 0, 0, 1, 1, 0):
        ds[i]["out"].fill_(3.0)
        graphs[i].replay()
        cases[i].check(ds[i])
        ws.fill_(0xFF)
