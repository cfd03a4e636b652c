"""fdkv_decode_parts on the GPU: shared prefixes, selected blocks, whole spans and
the exact tail in one softmax, against attention in 64 bits over the rows that the
cache's bytes hold, within the bound derived in serving_cases.  Caches start from
NaN bytes and tails hold NaN behind their rows, so a value that does not belong to
a sequence and reaches an output shows."""
import math
import sys

import numpy as np
import pytest

from serving_cases import attend, make_cache, unit_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


def log(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _dims(dtype, kv, G, d, k, sched=0, layers=None, ppm=None, rates=()):
    from paper_2607_06519_amd import binding as B
    layers = layers or {0: 2, 1: 12, 2: 4}[sched]
    if ppm is None and not rates:
        return B.dims(layers, kv, kv * G, d, k, dtype, sched)
    return B.dims(layers, kv, kv * G, d, 0, dtype, sched, B.RES_TOKENS, ppm or 0, rates)


def _modes(dims, n, seed):
    from paper_2607_06519_amd import binding as B
    rng = np.random.default_rng(seed)
    nb = len(B.blocks(dims)[0])
    m = np.stack([rng.permutation(np.resize([1, 0, 2, 1], nb * dims.n_kv_heads)) for _ in range(n)])
    m = m.reshape(n, nb, dims.n_kv_heads).astype(np.uint8)
    if dims.n_rates:
        m = np.where(m == 1, m | (rng.integers(0, dims.n_rates, m.shape) << 2).astype(np.uint8), m)
    return m


def _tail(torch, dims, batch, cap, lens, seed):
    """Tails [batch][Hkv][cap][d] of one layer with NaN behind their rows, and the lengths."""
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dims.dtype == 0 else torch.bfloat16
    k, v = (torch.randn(batch, dims.n_kv_heads, cap, dims.head_dim, generator=g).to(dt) for _ in range(2))
    for s, n in enumerate(lens):
        k[s, :, n:] = float("nan")
        v[s, :, n:] = float("nan")
    return k.cuda(), v.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()


class Case:
    """One call: shared caches, selected and whole spans, a tail; and what it has to give."""

    def __init__(self, torch, dims, dtype, batch, seed, shared=(), own=(), blocks=None, tail=None, qscale=2.0):
        from paper_2607_06519_amd import binding as B
        self.torch, self.dims, self.dtype, self.batch, self.B = torch, dims, dtype, batch, B
        self.G = dims.n_q_heads // dims.n_kv_heads
        self.shared = [make_cache(torch, dims, [T], _modes(dims, 1, seed + 3 * i), seed + i)[0] for i, T in enumerate(shared)]
        self.own = [make_cache(torch, dims, lens, _modes(dims, batch, seed + 50 + i), seed + 100 + i)[0] for i, lens in enumerate(own)]
        self.sel = None
        if blocks is not None:
            lens, lists, n_sel = blocks
            self.sel = make_cache(torch, dims, lens, _modes(dims, batch, seed + 70), seed + 200)[0]
            self.lists = lists                                 # [batch][Hkv] lists of block numbers
            host = np.full((batch, dims.n_kv_heads, n_sel), 1 << 30, np.int32)
            count = np.zeros((batch, dims.n_kv_heads), np.int32)
            for s in range(batch):
                for h in range(dims.n_kv_heads):
                    count[s, h] = len(lists[s][h])
                    host[s, h, :count[s, h]] = lists[s][h]
            self.blocks, self.counts, self.n_sel = torch.from_numpy(host).cuda(), torch.from_numpy(count).cuda(), n_sel
        self.tail_lens = tail[1] if tail else None
        self.tail = _tail(torch, dims, batch, tail[0], tail[1], seed + 9) if tail else None
        g = torch.Generator().manual_seed(seed + 11)
        dt = torch.float32 if dims.dtype == 0 else torch.bfloat16
        self.q = (qscale * torch.randn(batch, dims.n_q_heads, dims.head_dim, generator=g)).to(dt).cuda()
        self.scale = 1.0 / math.sqrt(dims.head_dim)
        self.parts = [B.part(B.PART_SHARED, c.seq_lens, c.max_seq_len, c.modes, c.offsets, c.buf) for c in self.shared]
        self.parts += [B.part(B.PART_OWN, c.seq_lens, c.max_seq_len, c.modes, c.offsets, c.buf) for c in self.own]
        if self.sel is not None:
            c = self.sel
            self.parts.append(B.part(B.PART_BLOCKS, c.seq_lens, c.max_seq_len, c.modes, c.offsets, c.buf, self.blocks,
                                     self.counts, self.n_sel))
        self.cap = tail[0] if tail else -1
        self.ws = torch.full((B.decode_parts_workspace(dims, batch, self.parts, self.cap) // 4 + 8,), float("nan"), device="cuda")

    def run(self, layer, out=None, stream=None):
        B = self.B
        out = self.torch.full_like(self.q, 7.0) if out is None else out
        tail = B.Tail(self.tail[2].data_ptr(), self.cap, self.tail[0].data_ptr(), self.tail[1].data_ptr()) if self.tail else None
        B.decode_parts(self.dims, self.batch, self.parts, tail, layer, self.q, out, self.scale, self.ws, stream)
        return out

    def want(self, layer):
        """Outputs and bounds [batch][Hq][d]."""
        dm, G = self.dims, self.G
        raw = {id(c): c.buf.cpu().numpy() for c in self.shared + self.own + ([self.sel] if self.sel else [])}
        q = self.q.double().cpu().numpy()
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        for h in range(dm.n_kv_heads):
            common = [unit_rows(c, raw[id(c)], 0, layer, h, self.dtype) for c in self.shared]
            for s in range(self.batch):
                parts = list(common) + [unit_rows(c, raw[id(c)], s, layer, h, self.dtype) for c in self.own]
                if self.sel is not None:
                    rows = unit_rows(self.sel, raw[id(self.sel)], s, layer, h, self.dtype)
                    T = len(rows[0])
                    for j in self.lists[s][h]:
                        if 0 <= j < -(-T // 64):
                            parts.append(tuple(r[64 * j:64 * j + 64] for r in rows))
                if self.tail:
                    n = self.tail_lens[s]
                    k, v = (self.tail[i][s, h, :n].double().cpu().numpy() for i in range(2))
                    parts.append((k, v, 0 * k, 0 * v))
                sl = slice(h * G, (h + 1) * G)
                out[s, sl], tol[s, sl] = attend(q[s, sl], parts, self.scale, self.dtype == "f32", True)
        return out, tol

    def check(self, layers=None, what=""):
        worst = 0.0
        for layer in layers if layers is not None else range(self.dims.n_layers):
            got = self.run(layer).double().cpu().numpy()
            out, tol = self.want(layer)
            assert np.isfinite(got).all(), (what, layer, np.argwhere(~np.isfinite(got))[:4])
            over = np.abs(got - out) - tol
            assert (over <= 0).all(), (what, layer, float(over.max()), np.argwhere(over > 0)[:4].tolist())
            norm = np.linalg.norm(out)
            worst = max(worst, np.linalg.norm(got - out) / norm if norm else 0.0)
        log(f"  {what}: worst rel-L2 {worst:.2e}")
        return worst


# dtype, d, G, k, schedule, layers looked at, ppm, rates
KINDS = {
    "bf16_pairs": ("bf16", 128, 4, 16, 0, None, None, ()),
    "bf16_pairs_k5": ("bf16", 128, 2, 5, 0, None, None, ()),
    "bf16_pairs_k128": ("bf16", 128, 8, 128, 0, (1,), None, ()),
    "bf16_pairs_k0_d64": ("bf16", 64, 1, 0, 0, None, None, ()),
    "bf16_quads_k24": ("bf16", 128, 4, 24, 2, None, None, ()),
    "bf16_quads_d64_k7": ("bf16", 64, 8, 7, 2, None, None, ()),
    "bf16_mixed": ("bf16", 128, 4, 16, 1, (0, 5, 11), None, ()),
    "e4m3_pairs": ("bf16_e4m3", 128, 4, 16, 0, None, None, ()),
    "e4m3_quads_d64": ("bf16_e4m3", 64, 2, 8, 2, None, None, ()),
    "e4m3_quads": ("bf16_e4m3", 128, 1, 16, 2, None, None, ()),
    "f32_pairs_d64": ("f32", 64, 2, 8, 0, None, None, ()),
    "f32_quads": ("f32", 128, 4, 24, 2, None, None, ()),
    "bf16_tokens": ("bf16", 128, 4, 0, 0, None, 60000, ()),
    "bf16_tokens_quads_many": ("bf16", 128, 2, 0, 2, None, 500000, ()),
    "bf16_tokens_none": ("bf16", 128, 4, 0, 0, None, 0, ()),
    "e4m3_tokens_quads_d64": ("bf16_e4m3", 64, 4, 0, 2, None, 100000, ()),
    "e4m3_tokens_all": ("bf16_e4m3", 128, 4, 0, 0, (1,), 1000000, ()),
    "f32_tokens_d64": ("f32", 64, 2, 0, 0, None, 100000, ()),
    "f32_tokens_quads": ("f32", 128, 1, 0, 2, None, 200000, ()),
    "bf16_rates": ("bf16", 128, 4, 0, 0, None, None, (10000, 100000, 400000)),
}


def _kind(name, kv=4):
    dtype, d, G, k, sched, layers, ppm, rates = KINDS[name]
    return _dims(dtype, kv, G, d, k, sched, None, ppm, rates), dtype, layers


@pytest.mark.parametrize("name", list(KINDS))
def test_shared_prefix(torch_dev, name):
    dims, dtype, layers = _kind(name)
    log(f"[case] shared {name}")
    for batch, T, tail in ((3, 333, (40, [0, 40, 17])), (5, 1, None), (2, 700, None)):
        Case(torch_dev, dims, dtype, batch, 1000 + T, shared=(T,), tail=tail).check(layers, f"{name} b{batch} T{T}")


@pytest.mark.parametrize("name", list(KINDS))
def test_selected_blocks(torch_dev, name):
    dims, dtype, layers = _kind(name)
    log(f"[case] blocks {name}")
    rng = np.random.default_rng(3)
    lens = [517, 64, 0, 1000]
    lists = [[sorted(rng.permutation(-(-T // 64))[:rng.integers(0, 7)].tolist()) for _ in range(dims.n_kv_heads)] for T in lens]
    lists[0][0] = [8, 0, 3]                # any order, the last block short
    lists[0][1] = []                       # nothing but the tail
    lists[3][0] = [-1, 15, 99, 2, 1 << 29] # numbers outside the sequence are passed over
    lists[3][1] = [5, 5, 15]               # a block listed twice counts twice
    Case(torch_dev, dims, dtype, 4, 77, blocks=(lens, lists, 9), tail=(70, [3, 70, 0, 33])).check(layers, name)


@pytest.mark.parametrize("batch,G,T", [(1, 1, 2048), (16, 1, 900), (17, 1, 900), (4, 8, 1300), (33, 1, 400), (16, 4, 1500), (9, 8, 500),
                                       (64, 4, 257), (70, 1, 130)])
def test_row_groups(torch_dev, batch, G, T):
    """Every number of column tiles and row groups, full and ragged."""
    dims = _dims("bf16", 2, G, 128, 16)
    log(f"[case] rows {batch} x {G}, T {T}")
    Case(torch_dev, dims, "bf16", batch, 5, shared=(T,), tail=(33, [(7 * s) % 34 for s in range(batch)])).check((1,), f"{batch}x{G}")


@pytest.mark.parametrize("dtype,G,batch", [("f32", 8, 9), ("bf16_e4m3", 8, 16), ("f32", 1, 20), ("bf16_e4m3", 4, 5)])
def test_row_groups_of_other_types(torch_dev, dtype, G, batch):
    for d in (64, 128):
        Case(torch_dev, _dims(dtype, 2, G, d, 8), dtype, batch, 6, shared=(300,), tail=(20, [s % 21 for s in range(batch)])).check((0,), f"{dtype} {d}")


@pytest.mark.parametrize("dtype", ["bf16", "f32", "bf16_e4m3"])
def test_a_step_of_everything(torch_dev, dtype):
    """Two shared spans, selected blocks, whole spans and the tail in one softmax."""
    dims = _dims(dtype, 3, 2, 128, 16)
    c = Case(torch_dev, dims, dtype, 4, 31, shared=(200, 513), own=([100, 0, 65, 31], [7, 0, 300, 1]),
             blocks=([400, 0, 130, 1], [[[1, 4]] * 3, [[]] * 3, [[0, 1, 2]] * 3, [[0]] * 3], 5), tail=(50, [9, 0, 50, 1]))
    c.check(None, dtype)


def test_long_chunks_and_many_parts(torch_dev):
    """A batch that fills the card (chunks at their longest) and as many parts as a call takes."""
    dims = _dims("bf16", 8, 1, 64, 8)
    Case(torch_dev, dims, "bf16", 64, 41, own=([9000] + [50] * 63,)).check((0,), "long chunk")
    dims = _dims("bf16", 2, 2, 64, 8)
    Case(torch_dev, dims, "bf16", 2, 43, shared=tuple(range(20, 160, 20)), own=tuple([40 + i, 0] for i in range(8)),
         tail=(20, [20, 0])).check((1,), "16 parts")


def test_long_prefix_and_sharp_queries(torch_dev):
    for dtype, qs in (("bf16", 8.0), ("f32", 8.0), ("bf16_e4m3", 30.0)):
        dims = _dims(dtype, 1, 4, 128, 16)
        Case(torch_dev, dims, dtype, 16, 51, shared=(12345,), tail=(8, [s % 9 for s in range(16)]), qscale=qs).check((1,), f"{dtype} q {qs}")


def test_rows_that_see_nothing(torch_dev):
    torch = torch_dev
    dims = _dims("bf16", 2, 4, 128, 16)
    c = Case(torch, dims, "bf16", 3, 61, shared=(0,), own=([0, 5, 0],), tail=(4, [0, 0, 2]))
    out = c.run(0)
    assert (out[0] == 0).all() and (out[1] != 0).any()
    c.check(None, "mostly empty")
    only = Case(torch, dims, "bf16", 2, 62)                      # no part at all
    assert (only.run(1) == 0).all()


def test_same_outputs_as_decode_spans(torch_dev):
    """Whole spans and a tail are fdkv_decode_spans; a shared span is as many copies of it."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    for dtype in ("bf16", "f32", "bf16_e4m3"):
        dims = _dims(dtype, 2, 4, 128, 16)
        c = Case(torch, dims, dtype, 3, 71, own=([700, 5, 64],), tail=(30, [30, 0, 2]))
        got = c.run(1).double()
        o = c.own[0]
        span = B.Span(o.seq_lens.data_ptr(), o.max_seq_len, o.modes.data_ptr(), o.offsets.data_ptr(), o.buf.data_ptr())
        ws = torch.empty(B.decode_spans_workspace(dims, 3, [o.max_seq_len], 30) // 4 + 8, device="cuda")
        ref = torch.empty_like(c.q)
        tail = B.Tail(c.tail[2].data_ptr(), 30, c.tail[0].data_ptr(), c.tail[1].data_ptr())
        B.decode_spans(dims, 3, [span], tail, 1, c.q, ref, c.scale, ws)
        _, tol = c.want(1)
        assert ((got - ref.double()).abs().cpu().numpy() <= 2 * tol).all(), dtype


def test_corrupt_units_come_out_nan(torch_dev):
    torch = torch_dev
    dims = _dims("bf16", 2, 4, 128, 16)
    for kind in ("mode", "offset"):
        c = Case(torch, dims, "bf16", 3, 81, shared=(300,), own=([70, 80, 90],), tail=(8, [8, 0, 3]))
        if kind == "mode":
            c.shared[0].modes[0, 0, 1] = 3
        else:
            c.own[0].offsets[2, 0, 0] += 128
        out = c.run(0).float().isnan()
        if kind == "mode":                                       # head 1 of every sequence
            assert out[:, 4:].all() and not out[:, :4].any()
        else:                                                    # head 0 of sequence 2
            assert out[2, :4].all() and not out[2, 4:].any() and not out[:2].any()


def test_graph_replays_and_side_streams(torch_dev):
    """A captured step replays with new contents of its inputs, and gives what the eager call gives; a call on a
    side stream too; two graphs with a workspace each do not meet."""
    torch = torch_dev
    dims = _dims("bf16", 2, 4, 128, 16)
    a = Case(torch, dims, "bf16", 4, 91, shared=(500,), blocks=([300, 64, 200, 1], [[[0, 2]] * 2, [[0]] * 2, [[1, 3]] * 2, [[0]] * 2], 4),
             tail=(30, [3, 30, 0, 9]))
    b = Case(torch, dims, "bf16", 4, 92, shared=(130,), tail=(30, [3, 30, 1, 9]))
    graphs, outs = [], []
    for c in (a, b):
        out = torch.zeros_like(c.q)
        c.run(1, out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run(1, out)
        graphs.append(g)
        outs.append(out)
    for step in range(4):
        for c in (a, b):
            c.q.copy_(torch.randn(c.q.shape, generator=torch.Generator().manual_seed(step)).to(c.q.dtype))
        a.tail[2].fill_(step + 1)
        a.tail[0].nan_to_num_(0.5), a.tail[1].nan_to_num_(0.25)
        for o in outs:
            o.fill_(9)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for c, o in zip((a, b), outs):
            assert torch.equal(o, c.run(1)), step
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(b.q)
    b.run(0, out, stream=side)
    side.synchronize()
    assert torch.equal(out, b.run(0))


def test_outputs_do_not_depend_on_padding(torch_dev):
    """Nothing around the output and the workspace is written."""
    torch = torch_dev
    dims = _dims("bf16", 2, 4, 128, 16)
    c = Case(torch, dims, "bf16", 5, 95, shared=(300,), tail=(8, [1, 2, 3, 0, 8]))
    n = c.q.numel()
    big = torch.full((n + 512,), 3.0, dtype=c.q.dtype, device="cuda")
    need = c.B.decode_parts_workspace(dims, 5, c.parts, 8)
    ws = torch.full((need // 4 + 256,), 5.0, device="cuda")
    whole, c.ws = ws, ws[:need // 4]
    c.run(0, big[256:256 + n].view_as(c.q))
    assert (big[:256] == 3).all() and (big[256 + n:] == 3).all() and (whole[need // 4:] == 5).all()
