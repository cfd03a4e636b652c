"""A serving step as a user runs it: Generation with a shared prefix, an indexed prefix
of its own whose blocks a step selects, and rows that are normed and rotated on their
way into the tail, eager, captured, and across a refresh.  Each operator's output is
checked against its formula in 64 bits on the very inputs that it got."""
import math

import numpy as np
import pytest

from serving_cases import attend, make_cache, unit_rows
from test_gpu_blocks import _want as blocks_want
from test_gpu_parts import _dims, _modes, log, torch_dev  # noqa: F401
from test_gpu_rope import _near, _want as rope_want

pytestmark = pytest.mark.gpu

EPS, FREQ = 1e-6, 10000.0


class Step:
    def __init__(self, torch, dtype, sched=0, batch=3, shared=300, lens=(1000, 64, 517), select=(1, 1, 4), cap=6, kv=2, G=4, d=128, k=16, ppm=None):
        from paper_2607_06519_amd import binding as B
        from paper_2607_06519_amd.cache import Generation
        self.torch, self.B, self.dtype, self.batch, self.G, self.cap = torch, B, dtype, batch, G, cap
        dims = self.dims = _dims(dtype, kv, G, d, k, sched, None, ppm)
        self.shared = make_cache(torch, dims, [shared], _modes(dims, 1, 3), 900)[0] if shared else None
        self.prefix = None
        if lens is not None:
            self.prefix, keys = make_cache(torch, dims, list(lens), _modes(dims, batch, 4), 901)
            if select is not None:
                for s, layers in enumerate(keys):
                    if layers is not None:
                        self.prefix.index(s, layers)
        self.select = select
        self.gen = Generation(dims, self.prefix, cap, shared=self.shared, select=select, batch=batch)
        g = self.g = torch.Generator().manual_seed(902)
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.freq = FREQ ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
        self.pos = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.rope = B.rope(d, self.freq.cuda(), self.pos)
        self.norm = [(1 + 0.2 * torch.randn(d, generator=g)).to(self.dt).cuda() for _ in range(2)]
        self.rows = torch.zeros(dims.n_layers, batch, (G + 2) * kv, d, dtype=self.dt, device="cuda")   # projections
        self.q, self.out = [None] * dims.n_layers, [None] * dims.n_layers
        self.picked = [None] * dims.n_layers

    def new_inputs(self, at):
        self.pos.copy_(self.torch.arange(self.batch, dtype=self.torch.int32) * 997 + at)
        self.rows.copy_(self.torch.randn(self.rows.shape, generator=self.g).to(self.dt))

    def run(self):
        dm = self.dims
        for l in range(dm.n_layers):
            q, k, v = self.rows[l].split((dm.n_q_heads, dm.n_kv_heads, dm.n_kv_heads), 1)
            self.q[l] = self.gen.append_rotated(l, self.rope, q, k, v, *self.norm, eps=EPS)
            self.out[l] = self.gen.decode(l, self.q[l])
            if self.select is not None:
                self.picked[l] = (self.gen.blocks.clone(), self.gen.counts.clone())

    def want(self, l, q, lists=None):
        """Outputs of layer ``l`` and their bounds [b][kv][G][d] for queries ``q``, over the cache as it is."""
        gen, num = self.gen, lambda t: t.double().cpu().numpy()
        n = gen.n_tail + 1
        raw = {id(c): c.buf.cpu().numpy() for c in [self.shared, *gen.spans] if c is not None}
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        for s in range(q.shape[0]):
            for h in range(q.shape[1]):
                have = [] if self.shared is None else [unit_rows(self.shared, raw[id(self.shared)], 0, l, h, self.dtype)]
                for i, c in enumerate(gen.spans):
                    rows = unit_rows(c, raw[id(c)], s, l, h, self.dtype)
                    if i == 0 and lists is not None:
                        have += [tuple(r[64 * j:64 * j + 64] for r in rows) for j in lists[s * q.shape[1] + h]]
                    else:
                        have.append(rows)
                k, v = (num(t[l][s, h, :n]) for t in (gen.tail_k, gen.tail_v))
                have.append((k, v, 0 * k, 0 * v))
                out[s, h], tol[s, h] = attend(q[s, h], have, 1.0 / math.sqrt(q.shape[-1]), self.dtype == "f32", True)
        return out, tol

    def check(self, what):
        dm, gen, f32 = self.dims, self.gen, self.dtype == "f32"
        num = lambda t: t.double().cpu().numpy()
        kv, G, d, b = dm.n_kv_heads, self.G, dm.head_dim, self.batch
        angle = self.pos.cpu().numpy().astype(np.float64)[:, None] * self.freq.numpy()
        n = gen.n_tail + 1
        for l in range(dm.n_layers):
            x = num(self.rows[l])
            y, m = rope_want(x[:, :kv * G], num(self.norm[0]), EPS, angle, d, 0)
            _near(num(self.q[l]), y, m, f32, d)
            y, m = rope_want(x[:, kv * G:kv * (G + 1)], num(self.norm[1]), EPS, angle, d, 0)
            _near(num(gen.tail_k[l][:, :, n - 1]), y, m, f32, d)
            assert np.array_equal(num(gen.tail_v[l][:, :, n - 1]), x[:, kv * (G + 1):])
            q = num(self.q[l]).reshape(b, kv, G, d)
            lists = None
            if self.select is not None:
                lists = blocks_want(num(self.prefix.bounds[l]), q, self.prefix.seq_lens_host, *self.select)
                got, count = (t.cpu().numpy() for t in self.picked[l])
                for i, w in enumerate(lists):
                    assert count.ravel()[i] == len(w) and got.reshape(b * kv, -1)[i, :len(w)].tolist() == w, (what, l, i)
            want, tol = self.want(l, q, lists)
            over = np.abs(num(self.out[l]).reshape(want.shape) - want) - tol
            assert (over <= 0).all(), (what, l, float(over.max()), np.argwhere(over > 0)[:4].tolist())


@pytest.mark.parametrize("dtype,sched,kw", [
    ("bf16", 0, {}), ("bf16_e4m3", 2, {}), ("f32", 0, dict(d=64, kv=3, G=2, k=5)), ("bf16", 2, dict(ppm=50000)),
    ("bf16", 0, dict(shared=0)), ("bf16", 0, dict(select=None)), ("bf16_e4m3", 0, dict(lens=None, select=None, batch=18)),
    ("bf16", 0, dict(lens=(130, 0, 900), select=(0, 0, 1))),
], ids=lambda x: "-".join(f"{k}{v}" for k, v in x.items()) if isinstance(x, dict) else str(x))
def test_steps(torch_dev, dtype, sched, kw):
    log(f"[case] steps {dtype} {sched} {kw}")
    st = Step(torch_dev, dtype, sched, **kw)
    for i in range(2):
        st.new_inputs(5000 + i)
        st.run()
        torch_dev.cuda.synchronize()
        st.check(f"step {i}")
        st.gen.advance()


@pytest.mark.parametrize("kw", [{}, dict(lens=None, select=None), dict(shared=0)], ids=["both", "shared", "selected"])
def test_refresh_and_the_steps_after(torch_dev, kw):
    """The tail becomes a span of its own, read whole beside the selected blocks and the shared prefix."""
    torch = torch_dev
    st = Step(torch, "bf16", cap=5, **kw)
    spans = len(st.gen.spans)
    for i in range(5):
        st.new_inputs(100 + i)
        st.run()
        st.gen.advance()
    assert st.gen.full
    with pytest.raises(RuntimeError):
        st.run()
    dm = st.dims
    probes = [torch.randn(st.batch, dm.n_q_heads, 4, dm.head_dim, generator=st.g).to(st.dt).cuda() for _ in range(dm.n_layers)]
    st.gen.refresh(probes, 4, lam=0.01)
    assert len(st.gen.spans) == spans + 1
    for i in range(2):
        st.new_inputs(105 + i)
        st.run()
        torch.cuda.synchronize()
        st.check(f"after the refresh, step {i}")
        st.gen.advance()


def test_captured_step(torch_dev):
    """All operators of a step in one graph, replayed with new rows, positions and tail lengths."""
    torch = torch_dev
    for dtype in ("bf16", "bf16_e4m3"):
        st = Step(torch, dtype)
        st.new_inputs(70)
        st.run()                                                  # (the library and its kernels are loaded)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            st.run()
        for i in range(4):
            st.new_inputs(70 + i)
            graph.replay()
            torch.cuda.synchronize()
            st.check(f"{dtype} replay {i}")
            kept = [o.clone() for o in st.out]
            eager = [st.gen.decode(l, st.q[l]) for l in range(st.dims.n_layers)]
            assert all(torch.equal(a, b) for a, b in zip(kept, eager))
            st.gen.advance()


def test_every_block_selected_is_the_whole_prefix(torch_dev):
    """n_sel of all blocks reads what the ordinary decode reads: no selection, no shared span."""
    torch = torch_dev
    from paper_2607_06519_amd.cache import Generation
    st = Step(torch, "bf16", shared=0, select=(0, 0, 16))
    plain = Generation(st.dims, st.prefix, st.cap)
    st.new_inputs(9)
    st.run()
    dm = st.dims
    for l in range(dm.n_layers):
        q, k, v = st.rows[l].split((dm.n_q_heads, dm.n_kv_heads, dm.n_kv_heads), 1)
        q = plain.append_rotated(l, st.rope, q, k, v, *st.norm, eps=EPS)
        assert torch.equal(q, st.q[l])
        assert torch.equal(plain.tail_k[l], st.gen.tail_k[l])
        apart = (st.out[l].double() - plain.decode(l, q).double()).abs().cpu().numpy()
        _, tol = st.want(l, q.double().cpu().numpy().reshape(st.batch, dm.n_kv_heads, st.G, dm.head_dim))
        assert (apart.reshape(tol.shape) <= 2 * tol).all()        # each within its bound of the exact output


def test_refusals(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd.cache import Generation
    st = Step(torch, "bf16")
    st.new_inputs(1)
    B, dm, gen = st.B, st.dims, st.gen
    q, k, v = st.rows[0].split((dm.n_q_heads, dm.n_kv_heads, dm.n_kv_heads), 1)
    for bad in (q.float(), q.cpu(), q[:, :-1], q[..., :64]):
        with pytest.raises(ValueError):
            gen.append_rotated(0, st.rope, bad, k, v)
    with pytest.raises(ValueError):
        gen.append_rotated(0, st.rope, q, k, v, st.norm[0].float())
    with pytest.raises(ValueError):
        gen.append_rotated(0, st.rope, q, k, v, st.norm[0][:64])
    good = torch.zeros(st.batch, dm.n_q_heads, dm.head_dim, dtype=st.dt, device="cuda")
    for bad in (good.float(), good.cpu(), good[:1], good.transpose(1, 2)):
        with pytest.raises(ValueError):
            gen.decode(0, bad)
    part = [B.part(B.PART_SHARED, st.shared.seq_lens, 300, st.shared.modes, st.shared.offsets, st.shared.buf)]
    with pytest.raises(ValueError):
        B.decode_parts(dm, st.batch, part, None, 0, good, good.float(), 1.0, gen._ws)
    with pytest.raises(ValueError):
        B.key_bounds(dm, 100, [torch.zeros(2, 99, 128, dtype=st.dt, device="cuda")] * 2, [torch.zeros(2, 2, 2, 128, dtype=st.dt, device="cuda")] * 2, 2)
    with pytest.raises(ValueError):
        B.block_select(dm, st.batch, st.prefix.seq_lens.long(), st.prefix.max_seq_len, st.prefix.bounds[0], good, 0, 0, 4, gen.blocks, gen.counts, gen._select_ws)
    c = st.shared
    for bad in (dict(seq_lens=c.seq_lens.long()), dict(modes=c.modes.int()), dict(seg_offsets=c.offsets.int()), dict(seq_lens=c.seq_lens.cpu())):
        with pytest.raises(ValueError):
            B.part(B.PART_SHARED, **{**dict(seq_lens=c.seq_lens, max_seq_len=300, modes=c.modes, seg_offsets=c.offsets, cache=c.buf), **bad})
    with pytest.raises(ValueError):
        B.rope(128, st.freq, st.pos)
    fresh = make_cache(torch, dm, [100] * st.batch, _modes(dm, st.batch, 1), 5)[0]
    for kw in (dict(prefix=fresh, select=(0, 1, 4)), dict(prefix=None), dict(prefix=None, shared=st.shared), dict(prefix=fresh, shared=fresh),
               dict(prefix=None, shared=st.shared, batch=2, select=(0, 0, 1)), dict(prefix=fresh, batch=7)):
        with pytest.raises(ValueError):
            Generation(dm, kw.pop("prefix"), 4, **kw)
    with pytest.raises(ValueError):
        gen.decode(0, good, sm_scale=-0.1)
    fresh.index(0, [torch.zeros(2, 100, 128, dtype=st.dt, device="cuda")] * 2)
    with pytest.raises(ValueError):                               # the other sequences have no bounds
        Generation(dm, fresh, 4, select=(0, 1, 4))
    with pytest.raises(B.FdkvError):
        Step(torch, "bf16", select=(3, 3, 4)).run()
