"""fdkv_prompt_attn over keys and values that are not finite: a token does not see those behind its own, whatever they
hold, against attention in 64 bits (bound: rows_cases)."""
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


CASES = [
    # dtype, d, kv, G, (query tokens, keys) of each sequence, keys of the first sequence whose rows are odd
    ("bf16", 128, 2, 1, [(130, 130)], [0, 31, 32, 63, 64, 65, 100, 129]),
    ("bf16", 128, 2, 4, [(200, 200), (33, 33)], [5, 6, 96, 127, 128, 191]),
    ("bf16", 128, 1, 8, [(70, 300), (3, 3)], [40, 230, 256, 299]),
    ("bf16", 64, 2, 2, [(150, 150), (9, 9)], [1, 62, 63, 64, 90, 149]),
    ("bf16", 64, 1, 1, [(64, 3001)], [2500, 2937, 2950, 2999]),    # keys split over workgroups
    ("bf16", 128, 1, 2, [(40, 4000)], [100, 3959, 3960, 3990]),
    ("f32", 64, 2, 2, [(101, 101), (40, 40)], [3, 31, 32, 33, 99, 100]),
    ("f32", 128, 1, 4, [(60, 700), (1, 1)], [641, 650, 672, 699]),
    ("bf16", 128, 64, 1, [(300, 300), (900, 900)], [7, 128, 170, 255, 299]),   # tiles of 32 keys
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:4])) + f"-{c[4][0]}")
@pytest.mark.parametrize("where", ["v", "k"])
def test_odd_rows(torch_dev, case, where):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dtype, d, kv, G, seqs, odd = case
    print(f"[case] odd {where} {case[:5]}", flush=True)
    g = torch.Generator().manual_seed(d + kv + G)
    f32, hq, dt = dtype == "f32", kv * G, torch.float32 if dtype == "f32" else torch.bfloat16
    dims, scale = B.dims(2, kv, hq, d, 0, dtype), 1.0 / math.sqrt(d)
    n, keys = sum(s[0] for s in seqs), [s[1] for s in seqs]
    starts, firsts = np.cumsum([0] + [s[0] for s in seqs]), np.cumsum([0] + keys)
    q = torch.randn(n, hq, d, generator=g).to(dt)
    K, V = (random_rows(torch, g, dtype, kv, sum(keys), d) for _ in range(2))
    values = [math.inf, -math.inf, math.nan]
    if where == "v":                                             # some channels of the rows
        for i, j in enumerate(odd):
            for h in range(kv):
                at = torch.randperm(d, generator=g)[:1 + 5 * i]
                V[h, j, at] = torch.tensor(values, dtype=dt)[(torch.arange(len(at)) + i) % 3]
    else:                                                        # keys and values that are no numbers at all
        K[:, odd] = math.nan
        V[:, odd] = math.nan
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()
    out = torch.full((n, hq, d), 7.0, dtype=dt, device="cuda")
    ws = torch.full((B.prompt_attn_workspace(dims, n, len(seqs), sum(keys)) // 4 + 64,), math.nan, device="cuda")
    B.prompt_attn(dims, q.cuda(), K[None].cuda(), V[None].cuda(), i32(starts), i32(keys), out, scale, ws, k_starts=i32(firsts[:-1]))
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    heads = range(hq) if hq <= 8 else (0, hq // 2 + 1, hq - 1)
    for s, (N, m) in enumerate(seqs):
        a, f = starts[s], firsts[s]
        seen = m - N + np.arange(N) + 1
        for h in heads:
            k, v = (x[h // G, f:f + m].double().numpy() for x in (K, V))
            o = got[a:a + N, h]
            if where == "k":
                good = seen <= min(odd) if s == 0 else np.ones(N, bool)
                assert np.isnan(o[~good]).all()
                fine = np.flatnonzero(good)
                want, bound = attend(q[a:a + N, h].double().numpy()[fine], np.nan_to_num(k), np.nan_to_num(v), scale, f32, seen[fine])
                check(o[fine], want, bound, (s, h))
                continue
            finite = np.isfinite(v)
            want, bound = attend(q[a:a + N, h].double().numpy(), k, np.where(finite, v, 0.0), scale, f32, seen)
            # what is not finite, of the keys that a token sees, by channel
            there = lambda mask: np.cumsum(mask, 0)[seen - 1] > 0
            up, down, no = there(v == math.inf), there(v == -math.inf), there(np.isnan(v))
            both = no | (up & down)
            assert np.isnan(o[both]).all() and (o[up & ~both] == math.inf).all() and (o[down & ~both] == -math.inf).all(), (s, h)
            rest = ~(up | down | no)
            assert np.isfinite(o[rest]).all() and (np.abs(o - want)[rest] <= bound[rest]).all(), (s, h)
