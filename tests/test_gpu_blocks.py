"""fdkv_key_bounds and fdkv_block_select on the GPU.  Bounds are keys' own values and
are compared as such; the selection is compared, number by number, with ranks
computed in 64 bits here (products of stored values are exact there, and the ranks of
random inputs lie far further apart than the order of a 64-bit sum can move them)."""
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


@pytest.mark.parametrize("dtype,d,kv,layers,T", [("bf16", 128, 8, 2, 1), ("bf16", 128, 2, 4, 64), ("bf16", 128, 3, 2, 65), ("bf16", 64, 2, 2, 1000),
                                                 ("f32", 64, 4, 2, 333), ("f32", 128, 1, 2, 511), ("bf16_e4m3", 128, 2, 2, 130)])
def test_key_bounds(torch_dev, dtype, d, kv, layers, T):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] bounds {dtype} d{d} kv{kv} L{layers} T{T}", flush=True)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(T)
    k = [torch.randn(kv, T, d, generator=g).to(dt) for _ in range(layers)]
    nb, cap = -(-T // 64), -(-T // 64) + 2
    out = torch.full((layers, kv, cap, 2, d), 9.0, dtype=dt, device="cuda")
    B.key_bounds(B.dims(layers, kv, kv, d, 0, dtype), T, [x.cuda() for x in k], list(out), cap)
    torch.cuda.synchronize()
    got = out.float().cpu()
    for l in range(layers):
        for j in range(nb):
            x = k[l][:, 64 * j:64 * j + 64].float()
            assert torch.equal(got[l, :, j, 0], x.amin(1)) and torch.equal(got[l, :, j, 1], x.amax(1)), (l, j)
    assert (got[:, :, nb:] == 9).all()


def _want(bounds, q, lens, first, last, n_sel):
    """Selected blocks per (sequence, KV head) from bounds [b][kv][nb][2][d] and q [b][kv][G][d] in float64."""
    out = []
    for s, T in enumerate(lens):
        nb = -(-T // 64)
        for h in range(bounds.shape[1]):
            lo, hi = bounds[s, h, :nb, 0], bounds[s, h, :nb, 1]
            if nb <= n_sel:
                out.append(list(range(nb)))
                continue
            rank = np.full(nb, -np.inf)
            for x in q[s, h]:
                u = np.maximum(x * lo, x * hi).sum(-1)
                rank = np.maximum(rank, u - u.max())
            ends = set(range(first)) | set(range(nb - last, nb))
            rest = sorted((j for j in range(nb) if j not in ends), key=lambda j: (-rank[j], j))
            out.append(sorted(ends) + rest[:n_sel - len(ends)])
    return [sorted(x) for x in out]


def _select(torch, B, dims, lens, bounds, q, first, last, n_sel):
    b, T = len(lens), max(lens)
    blocks = torch.full((b, dims.n_kv_heads, n_sel), -7, dtype=torch.int32, device="cuda")
    counts = torch.full((b, dims.n_kv_heads), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((B.block_select_workspace(dims, b, T) // 8 + 1,), float("nan"), dtype=torch.float64, device="cuda")
    B.block_select(dims, b, torch.tensor(lens, dtype=torch.int32).cuda(), T, bounds, q, first, last, n_sel, blocks, counts, ws)
    torch.cuda.synchronize()
    return blocks.cpu().numpy().reshape(-1, n_sel), counts.cpu().numpy().reshape(-1)


def _same(blocks, counts, want, n_sel):
    for i, w in enumerate(want):
        assert counts[i] == len(w), i
        assert blocks[i].tolist() == w + [-1] * (n_sel - len(w)), (i, blocks[i].tolist(), w)


@pytest.mark.parametrize("dtype,d,kv,G,lens,first,last,n_sel", [
    ("bf16", 128, 8, 4, [32768], 1, 2, 64),
    ("bf16", 128, 2, 8, [5000, 64, 0, 63, 2049], 0, 1, 9),
    ("bf16", 64, 3, 1, [3000, 700], 2, 4, 6),
    ("f32", 64, 2, 2, [4096, 1], 0, 0, 1),
    ("f32", 128, 1, 4, [9999], 1, 1, 128),
    ("bf16_e4m3", 128, 1, 2, [131072, 1000], 1, 4, 128),
    ("bf16", 128, 1, 1, [640], 0, 0, 10),
    ("bf16", 128, 1, 1, [641], 5, 5, 10),
])
def test_block_select(torch_dev, dtype, d, kv, G, lens, first, last, n_sel):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] select {dtype} d{d} kv{kv} G{G} {lens} sel {n_sel}", flush=True)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(sum(lens) + n_sel)
    cap = -(-max(lens) // 64)
    mid, rad = torch.randn(len(lens), kv, cap, d, generator=g), torch.rand(len(lens), kv, cap, d, generator=g)
    bounds = torch.stack([mid - rad, mid + rad], 3).to(dt)
    q = torch.randn(len(lens), kv, G, d, generator=g).to(dt)
    want = _want(bounds.double().numpy(), q.double().numpy(), lens, first, last, n_sel)
    for s, T in enumerate(lens):                                 # blocks behind a sequence hold anything
        bounds[s, :, -(-T // 64):] = float("nan")
    dims = B.dims(2, kv, kv * G, d, 0, dtype)
    _same(*_select(torch, B, dims, lens, bounds.cuda(), q.cuda(), first, last, n_sel), want, n_sel)


@pytest.mark.parametrize("kind", ["zero_query", "equal", "two_values", "steps", "huge", "one_apart"])
def test_ties_and_spreads(torch_dev, kind):
    """Many equal ranks (more than the list of a bin holds), ranks of very unlike size, and a lone outlier."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    nb, d, n_sel = 5000, 64, 100
    rng = np.random.default_rng(8)
    x = np.zeros((1, 1, nb, 2, d), np.float32)
    q = np.zeros((1, 1, 2, d), np.float32)
    q[..., 0, 0] = q[..., 1, 1] = 1
    if kind == "zero_query":
        q[:] = 0
        x[:] = rng.standard_normal(x.shape)
    elif kind == "equal":
        x[:] = 1
    elif kind == "two_values":
        x[0, 0, :, :, 0] = rng.integers(0, 2, (nb, 1)) * -1.0
        x[0, 0, :, :, 1] = -9
    elif kind == "steps":
        x[0, 0, :, :, 0] = -rng.integers(0, 40, (nb, 1))
        x[0, 0, :, :, 1] = -rng.integers(0, 40, (nb, 1))
    elif kind == "huge":
        x[0, 0, :, :, 0] = -np.exp2(rng.integers(-60, 100, (nb, 1)))
        x[0, 0, :, :, 1] = -3e38
    else:
        x[0, 0, :, :, 0] = -1 + 1e-6 * rng.random((nb, 1))
        x[0, 0, 77, :, 0] = 0
        x[0, 0, 78, :, 0] = -1e30
        x[0, 0, :, :, 1] = -1e35
    x[..., 0, :], x[..., 1, :] = np.minimum(x[..., 0, :], x[..., 1, :]), np.maximum(x[..., 0, :], x[..., 1, :])
    dims = B.dims(2, 1, 2, d, 0, "f32")
    for first, last in ((0, 0), (1, 3)):
        want = _want(x.astype(np.float64), q.astype(np.float64), [nb * 64], first, last, n_sel)
        _same(*_select(torch, B, dims, [nb * 64], torch.from_numpy(x).cuda(), torch.from_numpy(q).cuda(), first, last, n_sel), want, n_sel)


def test_captured_selection(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 2, 4, 64, 0, "bf16")
    g = torch.Generator().manual_seed(4)
    lens = torch.tensor([2000, 900], dtype=torch.int32).cuda()
    bounds = torch.randn(2, 2, 32, 2, 64, generator=g).sort(3)[0].to(torch.bfloat16).cuda()
    q = torch.randn(2, 4, 64, generator=g).to(torch.bfloat16).cuda()
    ws = torch.empty(B.block_select_workspace(dims, 2, 2000) // 8, dtype=torch.float64, device="cuda")
    make = lambda: (torch.empty(2, 2, 7, dtype=torch.int32, device="cuda"), torch.empty(2, 2, dtype=torch.int32, device="cuda"))
    out, eager = make(), make()
    call = lambda o: B.block_select(dims, 2, lens, 2000, bounds, q, 1, 1, 7, *o, ws)
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for step in range(4):
        q.copy_(torch.randn(2, 4, 64, generator=g).to(torch.bfloat16))
        lens[0] = 2000 - 300 * step
        graph.replay()
        torch.cuda.synchronize()
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1]), step


@pytest.mark.parametrize("what", ["nan_block", "inf_block", "all_nan", "inf_query"])
def test_selection_of_what_is_not_a_number(torch_dev, what):
    """Block numbers stay valid, ascending and distinct, whatever the bounds hold; the ends are among them."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] not a number: {what}", flush=True)
    T, n_sel = 6000, 20
    nb = -(-T // 64)
    bounds = torch.randn(1, 2, nb, 2, 128, generator=torch.Generator().manual_seed(1)).sort(3)[0].to(torch.bfloat16)
    q = torch.randn(1, 2, 4, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    if what == "nan_block":
        bounds[:, :, 7, :, 3] = float("nan")
    elif what == "inf_block":
        bounds[:, :, 7, 1, 3] = float("inf")
    elif what == "all_nan":
        bounds[:] = float("nan")
    else:
        q[:, :, 1, 5] = float("inf")
    blocks, counts = _select(torch, B, B.dims(2, 2, 8, 128, 0, "bf16"), [T], bounds.cuda(), q.cuda(), 1, 2, n_sel)
    assert (counts == n_sel).all()
    for row in blocks:
        assert (np.diff(row) > 0).all() and row[0] == 0 and row[-2:].tolist() == [nb - 2, nb - 1]
        if what == "nan_block":
            assert 7 not in row


def test_more_blocks_than_a_workgroup_holds(torch_dev):
    """Sequences of more than 4096 blocks keep their ranks in the workspace."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print("[case] 300000 tokens", flush=True)
    for dtype, d, G, lens, n_sel in (("bf16", 64, 4, [300000, 100], 100), ("f32", 64, 8, [262145, 262144], 4000), ("bf16", 128, 1, [600001], 1)):
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        g = torch.Generator().manual_seed(lens[0])
        cap = -(-max(lens) // 64)
        mid, rad = torch.randn(len(lens), 2, cap, d, generator=g), torch.rand(len(lens), 2, cap, d, generator=g)
        bounds = torch.stack([mid - rad, mid + rad], 3).to(dt)
        q = torch.randn(len(lens), 2, G, d, generator=g).to(dt)
        for first, last in ((0, 0), (0, 1)):
            want = _want(bounds.double().numpy(), q.double().numpy(), lens, first, last, n_sel)
            _same(*_select(torch, B, B.dims(2, 2, 2 * G, d, 0, dtype), lens, bounds.cuda(), q.cuda(), first, last, n_sel), want, n_sel)
    bounds[:] = bounds[:, :, :1]                                 # every rank alike: the lowest blocks
    want = [[0, 1, 2, 3, 9375]] * 2
    _same(*_select(torch, B, B.dims(2, 2, 2, d, 0, dtype), lens, bounds.cuda(), q.cuda(), 1, 1, 5), want, 5)
