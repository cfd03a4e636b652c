"""fdkv_rope_append on the GPU against its formulas in 64 bits.

The bound: y = x f w (f the norm), then a cos t - b sin t.  With u half an epsilon
of the element type and v = 2^-24, the sum of d squares is off by (d + 1) v of
itself, the norm by half of that and 4 v, a normed value by 3 v more; the angle's
fraction of a turn is rounded to fp32 (pi v), sine and cosine are off by at most 4 v;
two products and their sum add 3 v.  So y is off by at most
((d + 1) / 2 + 18) v (|a| + |b|), and rounded once: u |y|."""
import math
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


def _want(x, w, eps, angle, rot, inter):
    """x [n][heads][d] float64 -> rows and |a| + |b| of each value."""
    y = x.copy()
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * w
    mag = np.abs(y)
    z, m = y.copy(), mag.copy()
    if rot:
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        z[..., lo], z[..., hi] = y[..., lo] * c - y[..., hi] * s, y[..., hi] * c + y[..., lo] * s
        m[..., lo] = m[..., hi] = mag[..., lo] + mag[..., hi]
    return z, m


def _near(got, want, mag, f32, d):
    u, v = (2.0 ** -24 if f32 else 2.0 ** -8), 2.0 ** -24
    tol = u * np.abs(want) * 1.01 + ((d + 1) / 2 + 18) * v * mag
    over = np.abs(got - want) - tol
    assert (over <= 0).all(), (float(over.max()), np.argwhere(over > 0)[:4].tolist())


CASES = [
    # dtype, d, kv, G, n, rot, interleaved, axes, q norm, k norm
    ("bf16", 128, 8, 4, 1, 128, 0, 1, 0, 0),
    ("bf16", 128, 8, 4, 5, 128, 0, 1, 1, 1),
    ("bf16", 128, 2, 8, 37, 128, 1, 3, 1, 1),
    ("bf16", 64, 3, 2, 19, 32, 0, 2, 0, 1),
    ("bf16", 64, 1, 1, 7, 16, 1, 1, 1, 0),
    ("bf16", 128, 1, 1, 3, 0, 0, 1, 1, 1),
    ("bf16", 128, 5, 4, 1031, 96, 0, 3, 1, 1),
    ("bf16", 64, 2, 4, 1024, 64, 0, 1, 0, 0),
    ("f32", 64, 4, 2, 9, 64, 0, 1, 1, 1),
    ("f32", 128, 2, 4, 33, 48, 1, 4, 0, 0),
    ("f32", 128, 8, 1, 1029, 128, 0, 3, 1, 1),
    ("bf16_e4m3", 128, 2, 4, 4, 128, 0, 1, 1, 1),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_rope_append(torch_dev, case):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dtype, d, kv, G, n, rot, inter, axes, qn, kn = case
    print(f"[case] rope {case}", flush=True)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(n + d + rot)
    hq = kv * G
    dims = B.dims(2, kv, hq, d, 0, dtype)
    pad = 16                                                     # the fused rows are wider than their heads
    qkv = torch.randn(n, (hq + 2 * kv) * d + pad, generator=g).to(dt)
    q, k, v = qkv[:, :(hq + 2 * kv) * d].view(n, hq + 2 * kv, d).split((hq, kv, kv), 1)
    wq = (1 + 0.3 * torch.randn(d, generator=g)).to(dt) if qn else None
    wk = (1 + 0.3 * torch.randn(d, generator=g)).to(dt) if kn else None
    pos = torch.randint(-5, 1 << 20, (axes, n), generator=g).to(torch.int32)
    freq = 10000.0 ** (-torch.arange(0, max(rot, 2), 2, dtype=torch.float64) / max(rot, 2))
    axis = [i % axes for i in range(rot // 2)]
    batch, cap = (n, 11) if n < 64 else (3, n)
    seqs = torch.arange(n, dtype=torch.int32) if batch == n else torch.randint(3, (n,), generator=g).to(torch.int32)
    rows = torch.randint(cap, (n,), generator=g).to(torch.int32) if batch == n else torch.randperm(n, generator=g).to(torch.int32)
    skip = []
    if n > 4:                                                    # tokens with no place in the cache
        rows[1], rows[2], seqs[3] = -1, cap, -1
        seqs[4] = batch
        skip = [1, 2, 3, 4]
    dev = lambda t: None if t is None else t.cuda()
    dq = qkv.cuda()[:, :(hq + 2 * kv) * d].view(n, hq + 2 * kv, d).split((hq, kv, kv), 1)
    kc, vc = (torch.full((batch, kv, cap, d), 5.0, dtype=dt, device="cuda") for _ in range(2))
    qo = torch.full((n, hq, d), 7.0, dtype=dt, device="cuda")
    rope = B.rope(rot, dev(freq), dev(pos if axes > 1 else pos[0].contiguous()), axis, bool(inter))
    eps = 1e-5
    B.rope_append(dims, rope, *dq, qo, dev(seqs), dev(rows), kc, vc, dev(wq), dev(wk), eps)
    torch.cuda.synchronize()
    num = lambda t: None if t is None else t.double().cpu().numpy()
    angle = np.stack([pos[a].numpy().astype(np.float64) for a in (axis or [0])], 1) * freq.numpy()[:max(rot // 2, 1)]
    f32 = dtype == "f32"
    y, m = _want(num(q), num(wq), eps, angle, rot, inter)
    _near(num(qo), y, m, f32, d)
    y, m = _want(num(k), num(wk), eps, angle, rot, inter)
    gk, gv = num(kc), num(vc)
    used = np.zeros((batch, cap), bool)
    for i in range(n):
        if i in skip:
            continue
        s, r = int(seqs[i]), int(rows[i])
        used[s, r] = True
        _near(gk[s, :, r], y[i], m[i], f32, d)
        assert np.array_equal(gv[s, :, r], num(v[i]))
    assert (gk.transpose(0, 2, 1, 3)[~used] == 5).all() and (gv.transpose(0, 2, 1, 3)[~used] == 5).all()


def test_in_place_and_default_sequences(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 2, 8, 128, 0, "bf16")
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(6, h, 128, generator=g).to(torch.bfloat16).cuda() for h in (8, 2, 2))
    freq = (10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).cuda()
    pos = torch.arange(6, dtype=torch.int32).cuda() * 1000
    rope = B.rope(128, freq, pos)
    out, kc, vc = torch.empty_like(q), *(torch.zeros(6, 2, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = torch.tensor([0, 1, 2, 3, 0, 1], dtype=torch.int32).cuda()
    B.rope_append(dims, rope, q, k, v, out, None, rows, kc, vc)
    kc2, vc2 = torch.zeros_like(kc), torch.zeros_like(vc)
    B.rope_append(dims, rope, q, k, v, q, torch.arange(6, dtype=torch.int32).cuda(), rows, kc2, vc2)
    torch.cuda.synchronize()
    assert torch.equal(q, out) and torch.equal(kc, kc2) and torch.equal(vc, vc2)


def test_captured_step(torch_dev):
    """A captured call follows its positions and rows, replay after replay."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 2, 4, 64, 0, "f32")
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(3, h, 64, generator=g).cuda() for h in (4, 2, 2))
    freq = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).cuda()
    pos, rows = (torch.zeros(3, dtype=torch.int32).cuda() for _ in range(2))
    rope = B.rope(64, freq, pos)
    qo, kc, vc = torch.empty_like(q), *(torch.zeros(3, 2, 8, 64, device="cuda") for _ in range(2))
    B.rope_append(dims, rope, q, k, v, qo, None, rows, kc, vc)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rope_append(dims, rope, q, k, v, qo, None, rows, kc, vc)
    ek, ev, eq = torch.zeros_like(kc), torch.zeros_like(vc), torch.empty_like(qo)
    kc.zero_(), vc.zero_()
    for step in range(5):
        pos.fill_(100 * step)
        rows.fill_(step)
        q.mul_(1.5)
        graph.replay()
        B.rope_append(dims, rope, q, k, v, eq, None, rows, ek, ev)
        torch.cuda.synchronize()
        assert torch.equal(qo, eq) and torch.equal(kc, ek) and torch.equal(vc, ev), step
