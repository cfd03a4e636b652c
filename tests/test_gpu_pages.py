"""fdkv_page_write and fdkv_page_read on the GPU: rows bit for bit, FP8 rows against a search over the codes."""
import numpy as np
import pytest

from rows_cases import Pool, e4m3, held, random_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


@pytest.mark.parametrize("dtype,d,kv,page,n", [("bf16", 128, 8, 64, 1), ("bf16", 64, 3, 16, 100), ("f32", 128, 2, 32, 77), ("f32", 64, 1, 256, 300),
                                               ("bf16_e4m3", 128, 8, 64, 70), ("bf16_e4m3", 64, 2, 16, 333), ("bf16_e4m3", 128, 1, 128, 1)])
def test_rows_to_pages_and_back(torch_dev, dtype, d, kv, page, n):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] pages {dtype} d={d} kv={kv} page={page} n={n}", flush=True)
    g = torch.Generator().manual_seed(n + d)
    dims = B.dims(2, kv, kv, d, 0, dtype)
    lens = [n + 5, 40, 2 * page]
    pool = Pool(torch, dims, dtype, page, lens, seed=n)
    x = random_rows(torch, g, dtype, n, 2 * kv + 1, d)           # K and V of a fused projection's rows
    seqs = torch.randint(3, (n,), generator=g).to(torch.int32)
    rows = torch.zeros(n, dtype=torch.int32)
    for s in range(3):                                           # rows of a sequence in any order, each once
        at = torch.nonzero(seqs == s).flatten()
        take = torch.randperm(max(lens[s], len(at)), generator=g)[:len(at)].to(torch.int32)
        rows[at] = take
    cap = pool.table.shape[1] * page
    if n > 9:                                                    # tokens with no place
        seqs[1], seqs[2], rows[3], rows[4] = -1, 3, -1, cap
        rows[5], seqs[5] = cap - 1, 1                            # a page that is none
    ok = []
    for i in range(n):
        s, r = int(seqs[i]), int(rows[i])
        ok.append(0 <= s < 3 and 0 <= r < cap and int(pool.table[s, r // page]) >= 0)
    before = [t.clone() for t in (pool.k, pool.v)]
    xd = x.cuda()
    B.page_write(dims, pool.desc, xd[:, :kv], xd[:, kv:2 * kv], seqs.cuda(), rows.cuda())
    ko, vo = (torch.full((kv, n, d), 3.0, dtype=x.dtype, device="cuda") for _ in range(2))
    B.page_read(dims, pool.desc, ko.transpose(0, 1), vo.transpose(0, 1), seqs.cuda(), rows.cuda())
    torch.cuda.synchronize()
    for which, xs, got, old in (("k", x[:, :kv], ko, before[0]), ("v", x[:, kv:2 * kv], vo, before[1])):
        want = xs.double().numpy()
        if dtype == "bf16_e4m3":
            code, e = held(want)
            codes, exps = getattr(pool, which).cpu().numpy(), getattr(pool, which + "_exp").cpu().numpy()
            want = e4m3(code) * 2.0 ** (e.astype(np.float64) - 127)[..., None]
        got = got.double().cpu().numpy().transpose(1, 0, 2)
        now, was = (t.view(torch.uint8).cpu().numpy() for t in (getattr(pool, which), old))
        used = np.zeros(now.shape[:3], bool)
        for i in range(n):
            if not ok[i]:
                assert (got[i] == 3).all()
                continue
            page_id, slot = int(pool.table[int(seqs[i]), int(rows[i]) // page]), int(rows[i]) % page
            used[page_id, :, slot] = True
            assert np.array_equal(got[i], want[i]), (which, i)
            if dtype == "bf16_e4m3":
                assert np.array_equal(codes[page_id, :, slot], code[i]) and np.array_equal(exps[page_id, :, slot], e[i]), (which, i)
        assert np.array_equal(now[~used], was[~used])
        if dtype == "bf16_e4m3":
            assert (exps[~used] == 255).all()


def test_fp8_edges(torch_dev):
    """Rows of zeros, of one value, next to a step of the exponent, of subnormal numbers and of the largest ones."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    d = 64
    rows = []
    for top in (0.0, 448.0, 450.0, 446.0, 1.0, 1.75, 1.7578125, 7.0, 7.03125, 2.0 ** -133, 2.0 ** -126, 3.0 * 2.0 ** -130, 2.0 ** -120, 3.3895e38, 2.0 ** 127):
        r = np.linspace(-1, 1, d) * top
        r[0] = -top
        r[1:9] = top * np.array([2.0 ** -8, 17 / 16 * 2.0 ** -8, 2.0 ** -14, 2.0 ** -17, 2.0 ** -18, 1.5 * 2.0 ** -18, 2.0 ** -19, 0])
        rows.append(r)
    x = torch.tensor(np.array(rows)).to(torch.bfloat16).view(-1, 1, d)
    n = len(rows)
    dims = B.dims(2, 1, 1, d, 0, "bf16_e4m3")
    pool = Pool(torch, dims, "bf16_e4m3", 16, [n])
    at = torch.arange(n, dtype=torch.int32).cuda()
    out = [torch.empty(n, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.page_write(dims, pool.desc, x.cuda(), (-x).cuda(), torch.zeros_like(at), at)
    B.page_read(dims, pool.desc, *out, torch.zeros_like(at), at)
    torch.cuda.synchronize()
    for sign, t in zip((1, -1), out):
        code, e = held(sign * x.double().numpy())
        want = e4m3(code) * 2.0 ** (e.astype(np.float64) - 127)[..., None]
        want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)   # no bf16 number: 255 x 2^120 is held as 256 x 2^120
        bad = np.argwhere(t.double().cpu().numpy() != want)
        assert len(bad) == 0, bad[:5].tolist()


def test_values_that_are_not_finite(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    dims = B.dims(2, 1, 1, 64, 0, "bf16_e4m3")
    x = torch.ones(2, 1, 64, dtype=torch.bfloat16)
    x[0, 0, 3], x[1, 0, 5] = float("nan"), float("-inf")
    pool = Pool(torch, dims, "bf16_e4m3", 16, [1, 1])
    out = [torch.empty_like(x).cuda() for _ in range(2)]
    rows = torch.zeros(2, dtype=torch.int32).cuda()
    B.page_write(dims, pool.desc, x.cuda(), x.cuda(), None, rows)
    B.page_read(dims, pool.desc, *out, None, rows)
    torch.cuda.synchronize()
    for t in out:
        t = t.cpu()
        assert t[0, 0, 3].isnan() and t[1, 0, 5].isnan()
        assert (t[0, 0, [i for i in range(64) if i != 3]] == 1).all()


def test_strides_of_one(torch_dev):
    """One token, one head, one row: whatever the stride of that axis is."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    d, odd = 64, 2 ** 36 + 3
    dims = B.dims(2, 1, 4, d, 0, "bf16")
    pool = Pool(torch, dims, "bf16", 16, [1])
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    x, y, back = (torch.full((d,), f, dtype=torch.bfloat16, device="cuda") for f in (2.0, 3.0, 0.0))
    one = lambda t, *strides: t.as_strided((1,) * len(strides) + (d,), strides + (1,))
    B.page_write(dims, pool.desc, one(x, odd, odd), one(y, odd, d), i32(0), i32(0))
    B.page_read(dims, pool.desc, one(back, odd, odd), torch.empty(1, 1, d, dtype=torch.bfloat16, device="cuda"), i32(0), i32(0))
    q = torch.randn(4 * d, device="cuda").to(torch.bfloat16).as_strided((1, 4, d), (odd, d, 1))
    out = torch.empty(1, 4, d, dtype=torch.bfloat16, device="cuda")
    B.prompt_attn(dims, q, one(x, odd, odd, odd), one(y, odd, odd, odd), i32(0, 1), i32(1), out, 0.125,
                  torch.empty(max(1, B.prompt_attn_workspace(dims, 1, 1, 1)), dtype=torch.uint8, device="cuda"))
    assert (back == 2).all() and (out == 3).all()
