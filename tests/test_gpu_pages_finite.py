"""FP8 rows in pages with values that are not finite: those are held as NaN, and the row's other values as if they were
not there."""
import numpy as np
import pytest

from rows_cases import Pool, e4m3, held

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


@pytest.mark.parametrize("d", [64, 128])
def test_other_values_of_the_row(torch_dev, d):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] finite values beside others d={d}", flush=True)
    g = torch.Generator().manual_seed(d)
    inf, nan = float("inf"), float("nan")
    odd = [[], [inf], [-inf], [nan], [inf, -inf, nan], [-nan] * (d - 1), [inf] * d, [nan, -inf] * (d // 2)]
    n = len(odd)
    x = torch.randn(n, 2, d, generator=g).to(torch.bfloat16)
    for i, values in enumerate(odd):
        for h in range(2):
            at = torch.randperm(d, generator=g)[:len(values)]
            x[i, h, at] = torch.tensor(values, dtype=torch.bfloat16)
    dims = B.dims(2, 2, 2, d, 0, "bf16_e4m3")
    pool = Pool(torch, dims, "bf16_e4m3", 16, [n])
    rows = torch.arange(n, dtype=torch.int32).cuda()
    out = [torch.zeros_like(x).cuda() for _ in range(2)]
    B.page_write(dims, pool.desc, x.cuda(), (-x).cuda(), torch.zeros_like(rows), rows)
    B.page_read(dims, pool.desc, *out, torch.zeros_like(rows), rows)
    torch.cuda.synchronize()
    for sign, which, t in zip((1, -1), "kv", out):
        given = sign * x.double().numpy()
        finite = np.isfinite(given)
        code, e = held(np.where(finite, given, 0.0))
        page = int(pool.table[0, 0])
        codes, exps = (getattr(pool, name).cpu().numpy()[page, :, :n].swapaxes(0, 1) for name in (which, which + "_exp"))
        assert np.array_equal(exps, e)
        assert np.array_equal(codes[finite], code[finite]) and ((codes[~finite] & 127) == 127).all()
        want = np.where(finite, e4m3(code) * 2.0 ** (e.astype(np.float64) - 127)[..., None], np.nan)
        assert np.array_equal(t.double().cpu().numpy(), want, equal_nan=True)
