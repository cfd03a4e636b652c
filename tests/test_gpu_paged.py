"""fdkv_paged_attn on the GPU against attention in 64 bits over what the pages hold (bound: rows_cases)."""
import math

import numpy as np
import pytest

from rows_cases import Pool, attend, check, random_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


def fill(torch, pool, lens, seed):
    """Writes the first ``lens`` rows of every sequence (what lies behind them stays NaN)."""
    from paper_2607_06519_amd import binding as B
    g = torch.Generator().manual_seed(seed)
    for s, n in enumerate(lens):
        if n:
            kv, d = pool.dims.n_kv_heads, pool.dims.head_dim
            k, v = (random_rows(torch, g, pool.dtype, n, kv, d).cuda() for _ in range(2))
            rows = torch.arange(n, dtype=torch.int32).cuda()
            B.page_write(pool.dims, pool.desc, k, v, torch.full_like(rows, s), rows)
    torch.cuda.synchronize()


def _check(torch, pool, q, out, lens, scale, skip=()):
    """``skip``: (sequence, page of its table) that are passed over."""
    G = pool.dims.n_q_heads // pool.dims.n_kv_heads
    got, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
    for s, n in enumerate(lens):
        keep = np.ones(n, bool)
        for t, p in skip:
            if t == s:
                keep[p * pool.page:(p + 1) * pool.page] = False
        K, V = (pool.rows(w, s, n)[:, keep] if n else np.zeros((pool.dims.n_kv_heads, 0, pool.dims.head_dim)) for w in "kv")
        for h in range(pool.dims.n_kv_heads):
            want, bound = attend(qd[s, h * G:(h + 1) * G], K[h], V[h], scale, pool.dtype == "f32")
            check(got[s, h * G:(h + 1) * G], want, bound, (s, h))


CASES = [
    # dtype, d, kv, G, page, lengths, bound on them
    ("bf16", 128, 8, 4, 64, [1], 1),
    ("bf16", 128, 2, 8, 16, [0, 1, 15, 16, 17, 31, 32, 33], 33),
    ("bf16", 128, 1, 1, 128, [127, 128, 129, 500], 4000),
    ("bf16", 64, 3, 2, 32, [63, 1000, 64, 0], 1024),
    ("bf16", 64, 1, 4, 256, [3000], 3000),
    ("bf16", 128, 2, 4, 16, [4097, 5], 4097),
    ("bf16", 128, 1, 4, 16, [9000] * 2 + [1] * 40, 9000),
    ("bf16_e4m3", 128, 2, 4, 64, [1, 0, 77, 640], 640),
    ("bf16_e4m3", 64, 2, 8, 16, [33, 2050], 2050),
    ("bf16_e4m3", 128, 1, 2, 256, [5000], 5001),
    ("bf16_e4m3", 64, 1, 1, 32, [31, 32, 33], 64),
    ("f32", 64, 4, 2, 16, [1001, 7, 1, 300], 1001),
    ("f32", 128, 2, 4, 64, [65, 0, 2000], 2000),
    ("f32", 128, 1, 8, 32, [16, 17], 17),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:5])) + f"-{len(c[5])}-{c[6]}")
def test_paged_attn(torch_dev, case):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dtype, d, kv, G, page, lens, most = case
    print(f"[case] paged {case}", flush=True)
    dims = B.dims(2, kv, kv * G, d, 0, dtype)
    pool = Pool(torch, dims, dtype, page, [max(most, n) for n in lens], seed=d)
    fill(torch, pool, lens, 7)
    q = (1.5 * torch.randn(len(lens), kv * G, d, generator=torch.Generator().manual_seed(8))).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()
    ld = torch.tensor(lens, dtype=torch.int32).cuda()
    ws = torch.full((B.paged_attn_workspace(dims, len(lens), most) // 4,), math.nan, device="cuda")
    for scale in (1 / math.sqrt(d), -0.1, 0.0):
        out = torch.full_like(q, 9.0)
        B.paged_attn(dims, pool.desc, ld, most, q, out, scale, ws)
        torch.cuda.synchronize()
        _check(torch, pool, q, out, lens, scale)


@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3", "f32"])
def test_pages_that_are_none(torch_dev, dtype):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 2, 4, 128, 0, dtype)
    lens = [200, 40, 16]
    pool = Pool(torch, dims, dtype, 16, [200, 200, 200], seed=2)
    fill(torch, pool, lens, 3)
    skip = [(0, 0), (0, 3), (0, 12), (1, 1), (2, 0)]
    kept = pool.table.clone()
    for i, (s, p) in enumerate(skip):
        pool.table_d[s, p] = (-1, pool.n_pages, -5, 2147483647, -2147483648)[i]
    q = torch.randn(3, 4, 128, generator=torch.Generator().manual_seed(4)).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()
    out = torch.empty_like(q)
    ws = torch.empty(B.paged_attn_workspace(dims, 3, 200) // 4, device="cuda")
    B.paged_attn(dims, pool.desc, torch.tensor(lens, dtype=torch.int32).cuda(), 200, q, out, 0.1, ws)
    torch.cuda.synchronize()
    pool.table = kept
    _check(torch, pool, q, out, lens, 0.1, skip)
    assert (out[2] == 0).all()


def test_captured_steps(torch_dev):
    """A step captured once: a row appended and attended, replay after replay."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 2, 8, 128, 0, "bf16_e4m3")
    pool, other = (Pool(torch, dims, "bf16_e4m3", 16, [400, 400], seed=6) for _ in range(2))
    fill(torch, pool, [130, 250], 3)
    fill(torch, other, [130, 250], 3)
    g = torch.Generator().manual_seed(9)
    q = torch.randn(2, 8, 128, generator=g).to(torch.bfloat16).cuda()
    k, v = (random_rows(torch, g, "bf16", 2, 2, 128).cuda() for _ in range(2))
    rows = torch.tensor([130, 250], dtype=torch.int32).cuda()
    lens = rows + 1
    ws, ws2 = (torch.empty(B.paged_attn_workspace(dims, 2, 400) // 4, device="cuda") for _ in range(2))
    out, eager = torch.empty_like(q), torch.empty_like(q)

    def step(pool, out, ws):
        B.page_write(dims, pool.desc, k, v, None, rows)
        B.paged_attn(dims, pool.desc, lens, 400, q, out, 0.1, ws)
    step(pool, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pool, out, ws)
    for i in range(20):
        k.mul_(-1.125)
        q.add_(0.25)
        graph.replay()
        step(other, eager, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i
        rows.add_(1)
        lens.add_(1)
    assert torch.equal(pool.k, other.k) and torch.equal(pool.k_exp, other.k_exp)


@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3", "f32"])
@pytest.mark.parametrize("lens", [[0, 0, 0], [1, 200, 0], [3000, 10, 700]])
def test_behind_a_compressed_prefix(torch_dev, dtype, lens):
    """Records of a compressed prefix join in: the same as a decode over the prefix and a tail of the same rows."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    from serving_cases import attend as attend_parts, make_cache, unit_rows
    dims = B.dims(2, 2, 8, 128, 16, dtype)
    prefix = [700, 0, 90]
    modes = np.array([[[0, 1]], [[2, 0]], [[1, 2]]], np.uint8)
    cache, _ = make_cache(torch, dims, prefix, modes, 5)
    raw = cache.host_bytes()
    pool = Pool(torch, dims, dtype, 32, [max(lens + [1])] * 3, seed=6)
    fill(torch, pool, lens, 3)
    q = torch.randn(3, 8, 128, generator=torch.Generator().manual_seed(4)).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()
    out, most = torch.empty_like(q), max(lens)
    ws = torch.full((B.paged_attn_workspace(dims, 3, most) // 4,), math.nan, device="cuda")
    ld = torch.tensor(lens, dtype=torch.int32).cuda()
    for layer in range(2):
        B.decode_partial(dims, 3, cache.seq_lens, cache.max_seq_len, cache.modes, cache.offsets, cache.buf, layer, q, 0.1, cache.ws)
        B.paged_attn(dims, pool.desc, ld, most, q, out, 0.1, ws, more=cache.ws, n_more=2)
        torch.cuda.synchronize()
        got, qn = out.double().cpu().numpy(), q.double().cpu().numpy()
        for s in range(3):
            for h in range(2):
                held = [pool.rows(w, s, lens[s])[h] if lens[s] else np.zeros((0, 128)) for w in "kv"]
                parts = [unit_rows(cache, raw, s, layer, h, dtype), (*held, *(np.zeros_like(held[0]) for _ in range(2)))]
                want, bound = attend_parts(qn[s, 4 * h:4 * h + 4], parts, 0.1, dtype == "f32", False)
                check(got[s, 4 * h:4 * h + 4], want, bound, (layer, s, h))
