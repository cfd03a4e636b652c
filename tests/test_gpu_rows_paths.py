"""Paths of exact rows that sizes choose: calls whose workgroups all run at once (the first of them take tiles of query rows
from the last one on, the others from the first one on), joins of many records by their channels or by whole workgroups,
and every call on a stream of its own.  Against attention in 64 bits (bound: rows_cases)."""
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


def _prompt(torch, dtype, d, kv, G, seqs, heads, ws_bytes=None):
    """Packed prompts into an output of NaN; a sample of the heads checked.  ``seqs``: (query tokens, keys)."""
    from paper_2607_06519_amd import binding as B
    g = torch.Generator().manual_seed(d + kv + len(seqs))
    dt, hq = torch.float32 if dtype == "f32" else torch.bfloat16, kv * G
    dims = B.dims(2, kv, hq, d, 0, dtype)
    n, keys = sum(s[0] for s in seqs), [s[1] for s in seqs]
    q = torch.randn(n, hq, d, generator=g).to(dt).cuda()
    k, v = (random_rows(torch, g, dtype, 1, kv, sum(keys), d).cuda() for _ in range(2))
    starts, firsts = np.cumsum([0] + [s[0] for s in seqs]), np.cumsum([0] + keys)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()
    out = torch.full_like(q, math.nan)
    size = B.prompt_attn_workspace(dims, n, len(seqs), sum(keys))
    if ws_bytes is not None:
        assert size == ws_bytes(n * hq * (d + 4) * 4, size), size
    ws = torch.full((size // 4 + 64,), math.nan, device="cuda")
    B.prompt_attn(dims, q, k, v, i32(starts), i32(keys), out, 0.1, ws, k_starts=i32(firsts[:-1]))
    torch.cuda.synchronize()
    assert out.isfinite().all()
    got = out.double().cpu().numpy()
    for s, (N, m) in enumerate(seqs):
        a, f = starts[s], firsts[s]
        for h in heads:
            want, bound = attend(q[a:a + N, h].double().cpu().numpy(), k[0, h // G, f:f + m].double().cpu().numpy(),
                                 v[0, h // G, f:f + m].double().cpu().numpy(), 0.1, dtype == "f32", np.clip(m - N + np.arange(N) + 1, 0, m))
            check(got[a:a + N, h], want, bound, (s, h))


@pytest.mark.parametrize("dtype,d,kv,G,seqs", [
    ("bf16", 128, 8, 4, [(2048, 2048)]),
    ("bf16", 128, 8, 4, [(1001, 1001), (0, 7), (999, 1100)]),
    ("bf16", 128, 6, 2, [(4100, 4100)]),
    ("bf16", 64, 8, 8, [(700, 700), (0, 0), (1, 1), (300, 300)]),
    ("bf16", 64, 5, 1, [(7001, 7001)]),
    ("bf16", 128, 128, 2, [(100, 100), (65, 65)]),
    ("f32", 128, 8, 4, [(2048, 2048)]),
    ("f32", 64, 16, 2, [(2061, 2061)]),
])
def test_workgroups_that_run_at_once(torch_dev, dtype, d, kv, G, seqs):
    n = sum(s[0] for s in seqs)
    tiles = n * G // 128 + len(seqs)
    assert n * G // 128 * kv <= 512 and tiles > max(256 // kv, 1)  # (they all run at once, some from the first tile on)
    print(f"[case] at once {dtype} d={d} kv={kv} G={G} {seqs}", flush=True)
    _prompt(torch_dev, dtype, d, kv, G, seqs, (0, kv * G // 2, kv * G - 1), lambda record, size: 0)


@pytest.mark.parametrize("dtype,d,kv,G,seqs", [
    ("bf16", 64, 1, 1, [(3, 12001)]),
    ("bf16", 128, 1, 2, [(70, 10000), (1, 9000)]),
    ("bf16", 64, 2, 8, [(17, 20000)]),
    ("f32", 64, 1, 1, [(5, 3000)]),
    ("f32", 128, 2, 1, [(1, 700), (2, 1300)]),
])
def test_joins_of_many_splits(torch_dev, dtype, d, kv, G, seqs):
    print(f"[case] many splits {dtype} d={d} kv={kv} G={G} {seqs}", flush=True)

    def many(record, size):
        assert size % record == 0 and size // record > 8           # (whole workgroups join a row's records)
        return size
    _prompt(torch_dev, dtype, d, kv, G, seqs, range(kv * G), many)


def _fill(torch, pool, lens, stream=None):
    """Rows of every sequence, queued on ``stream``; the tensors that the calls read, to be kept until they are done."""
    from paper_2607_06519_amd import binding as B
    g, kept = torch.Generator().manual_seed(7), []
    for s, n in enumerate(lens):
        k, v = (random_rows(torch, g, pool.dtype, n, pool.dims.n_kv_heads, pool.dims.head_dim).cuda() for _ in range(2))
        rows = torch.arange(n, dtype=torch.int32).cuda()
        kept.append((k, v, torch.full_like(rows, s), rows))
    torch.cuda.synchronize()
    for x in kept:
        B.page_write(pool.dims, pool.desc, *x, stream=stream)
    return kept


@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3", "f32"])
@pytest.mark.parametrize("d,kv,G,lens", [(64, 1, 4, [5000]), (64, 2, 1, [3900]), (128, 1, 8, [5003]), (128, 2, 2, [4001, 100])])
def test_joins_by_channels(torch_dev, dtype, d, kv, G, lens):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] join {dtype} d={d} kv={kv} G={G} {lens}", flush=True)
    dims = B.dims(2, kv, kv * G, d, 0, dtype)
    most, batch = max(lens), len(lens)
    assert batch * kv * G <= 256 and -(-most // 128) > 24 and batch * kv * most <= 256 * 128   # (chunks of 128 tokens, 25 and more)
    pool = Pool(torch, dims, dtype, 32, lens, seed=d)
    _fill(torch, pool, lens)
    q = torch.randn(batch, kv * G, d, generator=torch.Generator().manual_seed(8)).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()
    out = torch.full_like(q, math.nan)
    ws = torch.full((B.paged_attn_workspace(dims, batch, most) // 4,), math.nan, device="cuda")
    B.paged_attn(dims, pool.desc, torch.tensor(lens, dtype=torch.int32).cuda(), most, q, out, 0.1, ws)
    torch.cuda.synchronize()
    got, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
    for s, n in enumerate(lens):
        K, V = (pool.rows(w, s, n) for w in "kv")
        for h in range(kv):
            want, bound = attend(qd[s, h * G:(h + 1) * G], K[h], V[h], 0.1, dtype == "f32")
            check(got[s, h * G:(h + 1) * G], want, bound, (s, h))


@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3", "f32"])
def test_every_call_on_its_stream(torch_dev, dtype):
    """Rows written, attended, read back and attended as a prompt's keys, in the order of each of two streams at once,
    give what they give on the current one."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] streams {dtype}", flush=True)
    dims, lens, n = B.dims(2, 2, 8, 128, 0, dtype), [900, 1500], 40
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(4)
    q = torch.randn(n, 8, 128, generator=g).to(dt).cuda()
    q2 = q[:2].contiguous()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    starts, k_lens, ld = i32(0, n), i32(lens[1]), i32(*lens)
    results = []
    for streams in ([None], [torch.cuda.Stream(), torch.cuda.Stream()]):
        state = []
        for stream in streams:
            pool = Pool(torch, dims, dtype, 32, lens, seed=3)
            state.append(dict(pool=pool, back=[torch.zeros(2, lens[1], 128, dtype=dt, device="cuda") for _ in range(2)],
                              step=torch.zeros_like(q2), prompt=torch.zeros_like(q),
                              ws=torch.zeros(max(B.paged_attn_workspace(dims, 2, lens[1]), B.prompt_attn_workspace(dims, n, 1, lens[1])) // 4 + 64,
                                             device="cuda")))
        torch.cuda.synchronize()
        kept = [_fill(torch, st["pool"], lens, stream) for st, stream in zip(state, streams)]
        for st, stream, given in zip(state, streams, kept):
            B.paged_attn(dims, st["pool"].desc, ld, lens[1], q2, st["step"], 0.1, st["ws"], stream=stream)
            B.page_read(dims, st["pool"].desc, *(x.transpose(0, 1) for x in st["back"]), *given[1][2:], stream=stream)
            B.prompt_attn(dims, q, *(x[None] for x in st["back"]), starts, k_lens, st["prompt"], 0.1, st["ws"], stream=stream)
        torch.cuda.synchronize()
        results += [[st["step"], st["prompt"], *st["back"], st["pool"].k, st["pool"].v] for st in state]
    for other in results[1:]:
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(results[0], other))
    assert results[0][0].isfinite().all() and results[0][1].isfinite().all() and (results[0][1] != 0).any()
