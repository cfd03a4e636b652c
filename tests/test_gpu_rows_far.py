"""Exact rows whose places pass 32 bits: pools of more than 4 GB, keys behind more than 4 GB of others, and calls on streams
of their own."""
import math

import numpy as np
import pytest

from rows_cases import Pool, attend, check, e4m3, held, random_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3"])
def test_pages_of_a_large_pool(torch_dev, dtype):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    kv, d, page = 8, 128, 256
    size = 2 if dtype == "bf16" else 1
    n_pages = ((1 << 32) + (1 << 29)) // (kv * page * d * size)
    dims = B.dims(2, kv, 4 * kv, d, 0, dtype)
    dt = torch.bfloat16 if dtype == "bf16" else torch.uint8
    print(f"[case] pool {dtype} {n_pages} pages", flush=True)
    k, v = (torch.empty(n_pages, kv, page, d, dtype=dt, device="cuda") for _ in range(2))
    exps = [torch.empty(n_pages, kv, page, dtype=torch.uint8, device="cuda") if size == 1 else None for _ in range(2)]
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2], [n_pages // 2, n_pages - 3, 1]], dtype=torch.int32).cuda()
    pages = B.pages(dims, k, v, table, *exps)
    g = torch.Generator().manual_seed(1)
    lens, rows_in = [700, 513], []
    for s, n in enumerate(lens):
        x = [random_rows(torch, g, dtype, n, kv, d) for _ in range(2)]
        at = torch.arange(n, dtype=torch.int32).cuda()
        B.page_write(dims, pages, x[0].cuda(), x[1].cuda(), torch.full_like(at, s), at)
        out = [torch.zeros(n, kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        B.page_read(dims, pages, *out, torch.full_like(at, s), at)
        torch.cuda.synchronize()
        want = [t.double().numpy() for t in x]
        if size == 1:
            want = [e4m3(c) * 2.0 ** (e.astype(np.float64) - 127)[..., None] for c, e in map(held, want)]
        assert all(np.array_equal(t.double().cpu().numpy(), w) for t, w in zip(out, want))
        rows_in.append(want)
    q = torch.randn(2, 4 * kv, d, generator=g).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    ws = torch.empty(B.paged_attn_workspace(dims, 2, 700) // 4, device="cuda")
    B.paged_attn(dims, pages, torch.tensor(lens, dtype=torch.int32).cuda(), 700, q, out, 0.1, ws)
    torch.cuda.synchronize()
    for s in range(2):
        for h in range(kv):
            want, bound = attend(q[s, 4 * h:4 * h + 4].double().cpu().numpy(), rows_in[s][0][:, h], rows_in[s][1][:, h], 0.1, False)
            check(out[s, 4 * h:4 * h + 4].double().cpu().numpy(), want, bound, (s, h))


def test_keys_behind_many_others(torch_dev):
    """Packed rows and a cache of sequences, both past 4 GB."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    kv, G, d, n = 2, 4, 128, 150
    dims = B.dims(2, kv, kv * G, d, 0, "bf16")
    g = torch.Generator().manual_seed(2)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    q = torch.randn(n, kv * G, d, generator=g).to(torch.bfloat16).cuda()
    K, V = (random_rows(torch, g, "bf16", kv, n, d).cuda() for _ in range(2))
    rows = (1 << 32) // (d * 2) + 1000                           # of a head: more than 4 GB
    outs = []
    for layout in ("packed", "cache"):
        print(f"[case] far {layout}", flush=True)
        shape = (1, kv, rows, d) if layout == "packed" else (3, kv, rows // 4, d)
        k, v = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        out = torch.empty_like(q)
        if layout == "packed":
            first = rows - n
            k[0, :, first:], v[0, :, first:] = K, V
            args = dict(q_starts=i32(0, n), k_lens=i32(n), k_starts=i32(first))
        else:
            k[2, :, :n], v[2, :, :n] = K, V
            args = dict(q_starts=i32(0, 0, 0, n), k_lens=i32(0, 0, n))
        ws = torch.empty(B.prompt_attn_workspace(dims, n, len(args["k_lens"]), shape[2]) // 4 + 64, device="cuda")
        B.prompt_attn(dims, q, k, v, out=out, sm_scale=0.1, ws=ws, **args)
        torch.cuda.synchronize()
        outs.append(out.double().cpu().numpy())
        del k, v
    for out in outs:
        for h in range(kv * G):
            want, bound = attend(q[:, h].double().cpu().numpy(), K[h // G].double().cpu().numpy(), V[h // G].double().cpu().numpy(), 0.1, False, np.arange(n) + 1)
            check(out[:, h], want, bound, h)


def test_streams(torch_dev):
    """Calls on two streams of their own, each with its workspace, give what calls in turn give."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 2, 8, 128, 0, "bf16_e4m3")
    g = torch.Generator().manual_seed(3)
    n, most = 60, 3000
    pools = [Pool(torch, dims, "bf16_e4m3", 32, [most, most], seed=s) for s in range(2)]
    q = torch.randn(2, n, 8, 128, generator=g).to(torch.bfloat16).cuda()
    k, v = (random_rows(torch, g, "bf16", 2, 1, 2, most, 128).cuda() for _ in range(2))
    rows = torch.arange(most, dtype=torch.int32).cuda()
    lens = torch.tensor([most, most], dtype=torch.int32).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()
    starts, klen = i32(0, n), i32(most)
    outs = [[torch.empty_like(q[0]) for _ in range(2)] for _ in range(2)]
    steps = [[torch.empty(2, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    ws = [[torch.empty(B.prompt_attn_workspace(dims, n, 1, most) // 4 + 64, device="cuda"),
           torch.empty(B.paged_attn_workspace(dims, 2, most) // 4 + 64, device="cuda")] for _ in range(2)]
    both = [torch.zeros_like(rows), torch.ones_like(rows)]

    def work(i, turn, stream):
        B.prompt_attn(dims, q[i], k[i], v[i], starts, klen, outs[turn][i], 0.1, ws[i][0], stream=stream)
        for s in both:
            B.page_write(dims, pools[i].desc, k[i][0].transpose(0, 1), v[i][0].transpose(0, 1), s, rows, stream=stream)
        B.paged_attn(dims, pools[i].desc, lens, most, q[i][:2].contiguous(), steps[turn][i], 0.1, ws[i][1], stream=stream)
    q2 = [q[i][:2].contiguous() for i in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        work(i, 0, None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i in range(2):
            B.prompt_attn(dims, q[i], k[i], v[i], starts, klen, outs[1][i], 0.1, ws[i][0], stream=streams[i])
            B.paged_attn(dims, pools[i].desc, lens, most, q2[i], steps[1][i], 0.1, ws[i][1], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[0][i], outs[1][i]) and torch.equal(steps[0][i], steps[1][i])
