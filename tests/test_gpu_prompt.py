"""fdkv_prompt_attn on the GPU against attention in 64 bits (bound: rows_cases)."""
import math

import numpy as np
import pytest

from rows_cases import attend, check, random_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


def _run(torch, dtype, d, kv, G, seqs, layout, scale=None, lead=0, trail=0, seed=1):
    """``seqs``: (query tokens, keys) of each sequence.  Rows that no sequence names hold NaN."""
    from paper_2607_06519_amd import binding as B
    print(f"[case] prompt {dtype} d={d} kv={kv} G={G} {seqs[:6]} {layout}", flush=True)
    g = torch.Generator().manual_seed(seed)
    f32, hq = dtype == "f32", kv * G
    dt = torch.float32 if f32 else torch.bfloat16
    dims = B.dims(2, kv, hq, d, 0, dtype)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    n = lead + sum(s[0] for s in seqs) + trail
    starts = np.cumsum([lead] + [s[0] for s in seqs])
    keys = [s[1] for s in seqs]
    K, V = ([random_rows(torch, g, dtype, kv, m, d) for m in keys] for _ in range(2))
    q = (1.5 * torch.randn(n, hq, d, generator=g)).to(dt)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()
    k_starts, gap = None, 3
    if layout == "cache":                                        # [batch][Hkv][cap][d]
        cap = max(keys) + gap
        kd, vd = (torch.full((len(seqs), kv, cap, d), math.nan, dtype=dt) for _ in range(2))
        for s, m in enumerate(keys):
            kd[s, :, :m], vd[s, :, :m] = K[s], V[s]
        kd, vd = kd.cuda(), vd.cuda()
    else:
        k_starts = np.cumsum([gap] + [m + gap for m in keys])[:-1]
        total = int(k_starts[-1]) + keys[-1] + gap
        kp, vp = (torch.full((kv, total, d), math.nan, dtype=dt) for _ in range(2))
        for s, m in enumerate(keys):
            kp[:, k_starts[s]:k_starts[s] + m], vp[:, k_starts[s]:k_starts[s] + m] = K[s], V[s]
        if layout == "packed":                                   # [Hkv][n][d]
            kd, vd = kp.cuda()[None], vp.cuda()[None]
        else:                                                    # a fused projection's rows [n][2 Hkv + 1][d]
            rows = torch.full((total, 2 * kv + 1, d), math.nan, dtype=dt)
            rows[:, :kv], rows[:, kv:2 * kv] = kp.transpose(0, 1), vp.transpose(0, 1)
            rows = rows.cuda()
            kd, vd = (rows[:, a:a + kv].transpose(0, 1)[None] for a in (0, kv))
    qd = q.cuda()
    if layout == "fused":                                        # queries between other heads
        wide = torch.full((n, hq + 2, d), math.nan, dtype=dt, device="cuda")
        wide[:, 1:1 + hq] = qd
        qd = wide[:, 1:1 + hq]
    out = torch.full((n, hq, d), 7.0, dtype=dt, device="cuda")
    ws = torch.full((B.prompt_attn_workspace(dims, n, len(seqs), kd.shape[2]) // 4 + 64,), math.nan, device="cuda")
    B.prompt_attn(dims, qd, kd, vd, i32(starts), i32(keys), out, scale, ws, k_starts=None if k_starts is None else i32(k_starts))
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    for s, (N, m) in enumerate(seqs):
        a = starts[s]
        for h in range(hq):
            seen = np.clip(m - N + np.arange(N) + 1, 0, m)
            want, bound = attend(q[a:a + N, h].double().numpy(), K[s][h // G].double().numpy(), V[s][h // G].double().numpy(), scale, f32, seen)
            check(got[a:a + N, h], want, bound, (s, h))
    assert (got[:lead] == 7).all() and (got[n - trail:] == 7).all()
    return out


CASES = [
    ("bf16", 128, 1, 1, [(1, 1)], "cache"),
    ("bf16", 128, 2, 4, [(64, 64)], "packed"),
    ("bf16", 128, 8, 4, [(129, 129)], "packed"),
    ("bf16", 128, 2, 8, [(33, 65), (1, 200), (7, 7)], "cache"),
    ("bf16", 128, 1, 2, [(128, 128), (0, 5), (63, 63), (65, 65), (0, 0), (5, 0)], "packed"),
    ("bf16", 128, 3, 1, [(300, 300), (31, 500)], "fused"),
    ("bf16", 64, 2, 4, [(257, 257), (2, 2), (40, 129)], "packed"),
    ("bf16", 64, 5, 1, [(1, 63), (1, 64), (1, 65), (3, 1000)], "cache"),
    ("bf16", 64, 1, 8, [(100, 100)], "fused"),
    ("bf16_e4m3", 128, 2, 2, [(70, 70)], "packed"),
    ("bf16", 128, 2, 4, [(10, 4), (40, 39), (9, 0)], "cache"),     # more tokens than keys: the first see none
    ("bf16", 128, 2, 4, [(600, 1111)], "cache"),
    ("bf16", 128, 1, 1, [(1, 5000)], "cache"),                     # keys split over workgroups
    ("bf16", 64, 2, 8, [(17, 3001), (2, 40)], "packed"),
    ("f32", 64, 4, 2, [(301, 301)], "packed"),
    ("f32", 128, 2, 4, [(33, 33), (1, 1), (0, 3), (90, 222)], "cache"),
    ("f32", 64, 1, 8, [(20, 2000), (5, 3)], "fused"),
    ("f32", 128, 1, 1, [(1, 1500), (64, 64)], "packed"),
    ("bf16", 128, 1, 1, [(1, 1)] * 70 + [(3, 9)] * 70, "packed"),  # more sequences than lanes
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:4])) + f"-{len(c[4])}-{c[4][-1]}-{c[5]}")
def test_prompt_attn(torch_dev, case):
    _run(torch_dev, *case, seed=len(case[4]) + case[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.5])
def test_scales(torch_dev, dtype, scale):
    _run(torch_dev, dtype, 64, 2, 2, [(70, 70), (5, 90)], "packed", scale=scale)


def test_tokens_of_no_sequence(torch_dev):
    _run(torch_dev, "bf16", 128, 2, 4, [(37, 37), (9, 30)], "packed", lead=5, trail=11)
    _run(torch_dev, "bf16", 128, 1, 1, [(2, 3000)], "cache", lead=3, trail=2)


def test_one_long_prompt(torch_dev):
    _run(torch_dev, "bf16", 128, 1, 2, [(1500, 1500)], "packed")


@pytest.mark.parametrize("dtype,d,kv,G,seqs", [
    ("bf16", 128, 16, 8, [(1100, 1100)]),                          # many workgroups: shorter tiles
    ("bf16", 128, 64, 1, [(700, 700), (1, 1), (1300, 1333), (33, 31)]),
    ("bf16", 64, 32, 4, [(900, 1000), (200, 200)]),
    ("f32", 64, 16, 4, [(2100, 2100)]),
])
def test_many_workgroups(torch_dev, dtype, d, kv, G, seqs):
    """A sample of the heads of a call that fills the card several times over."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, kv, kv * G, d, 0, dtype)
    g = torch.Generator().manual_seed(kv + G)
    n, keys = sum(s[0] for s in seqs), [s[1] for s in seqs]
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q = torch.randn(n, kv * G, d, generator=g).to(dt).cuda()
    total = sum(keys)
    k, v = (random_rows(torch, g, dtype, 1, kv, total, d).cuda() for _ in range(2))
    starts, firsts = np.cumsum([0] + [s[0] for s in seqs]), np.cumsum([0] + keys)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()
    out = torch.full_like(q, math.nan)
    B.prompt_attn(dims, q, k, v, i32(starts), i32(keys), out, 0.1, None, k_starts=i32(firsts[:-1]))
    torch.cuda.synchronize()
    assert out.isfinite().all()
    got = out.double().cpu().numpy()
    for s, (N, m) in enumerate(seqs):
        a, f = starts[s], firsts[s]
        for h in (0, kv * G // 2 + 1, kv * G - 1):
            want, bound = attend(q[a:a + N, h].double().cpu().numpy(), k[0, h // G, f:f + m].double().cpu().numpy(),
                                 v[0, h // G, f:f + m].double().cpu().numpy(), 0.1, dtype == "f32", np.clip(m - N + np.arange(N) + 1, 0, m))
            check(got[a:a + N, h], want, bound, (s, h))


def test_no_keys_at_all(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 2, 8, 128, 0, "bf16")
    q = torch.ones(5, 8, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.empty(1, 2, 0, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 3.0)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    B.prompt_attn(dims, q, k, k, i32(0, 4), i32(7), out, 0.1, None)
    torch.cuda.synchronize()
    assert (out[:4] == 0).all() and (out[4] == 3).all()


def test_in_place(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    g = torch.Generator().manual_seed(3)
    dims = B.dims(2, 2, 8, 128, 0, "bf16")
    q = torch.randn(200, 8, 128, generator=g).to(torch.bfloat16).cuda()
    k, v = (random_rows(torch, g, "bf16", 1, 2, 200, 128).cuda() for _ in range(2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    ws = torch.empty(B.prompt_attn_workspace(dims, 200, 1, 200) // 4 + 64, device="cuda")
    out = torch.empty_like(q)
    B.prompt_attn(dims, q, k, v, i32(0, 200), i32(200), out, 0.1, ws)
    B.prompt_attn(dims, q, k, v, i32(0, 200), i32(200), q, 0.1, ws)
    torch.cuda.synchronize()
    assert torch.equal(q, out)


def test_lengths_out_of_range(torch_dev):
    """Numbers outside of their ranges are taken as the nearest in them: nothing is read or written elsewhere."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    g = torch.Generator().manual_seed(4)
    dims = B.dims(2, 1, 2, 64, 0, "bf16")
    q = torch.randn(40, 2, 64, generator=g).to(torch.bfloat16).cuda()
    k, v = (random_rows(torch, g, "bf16", 1, 1, 100, 64).cuda() for _ in range(2))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    ws = torch.empty(B.prompt_attn_workspace(dims, 40, 2, 100) // 4 + 64, device="cuda")
    outs = []
    for starts, lens, first in ((i32(-7, 25, 99), i32(30, 500), i32(-4, 60)), (i32(0, 25, 40), i32(30, 40), i32(0, 60))):
        outs.append(torch.empty_like(q))
        B.prompt_attn(dims, q, k, v, starts, lens, outs[-1], 0.1, ws, k_starts=first)
    torch.cuda.synchronize()
    assert torch.equal(*outs)


def test_captured(torch_dev):
    """A captured call follows its lengths, replay after replay."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    g = torch.Generator().manual_seed(5)
    dims = B.dims(2, 2, 8, 128, 0, "bf16")
    q = torch.randn(30, 8, 128, generator=g).to(torch.bfloat16).cuda()
    k, v = (random_rows(torch, g, "bf16", 1, 2, 4000, 128).cuda() for _ in range(2))
    starts, lens = torch.tensor([0, 30], dtype=torch.int32).cuda(), torch.tensor([30], dtype=torch.int32).cuda()
    n = B.prompt_attn_workspace(dims, 30, 1, 4000)
    assert n > 0
    ws, ws2 = (torch.empty(n // 4, device="cuda") for _ in range(2))
    out, eager = torch.empty_like(q), torch.empty_like(q)
    B.prompt_attn(dims, q, k, v, starts, lens, out, 0.1, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.prompt_attn(dims, q, k, v, starts, lens, out, 0.1, ws)
    for m in (30, 31, 700, 3999, 0, 4000):
        lens.fill_(m)
        out.fill_(5)
        graph.replay()
        B.prompt_attn(dims, q, k, v, starts, lens, eager, 0.1, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, eager), m
