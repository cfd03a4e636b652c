"""PagedCache behind a compressed prefix from the first step on: the new token takes part, step after step."""
import math

import numpy as np
import pytest

from rows_cases import check, random_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3", "f32"])
def test_first_steps(torch_dev, dtype, captured):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    from paper_2607_06519_amd.cache import PagedCache
    from serving_cases import attend as attend_parts, make_cache, unit_rows
    print(f"[case] first steps {dtype} captured={captured}", flush=True)
    dims = B.dims(2, 2, 8, 128, 16, dtype)
    prefix, _ = make_cache(torch, dims, [300, 0, 600], np.array([[[0, 1]], [[0, 0]], [[2, 1]]], np.uint8), 3)
    raw = prefix.host_bytes()
    c = PagedCache(dims, 3, 100, page=16)
    g = torch.Generator().manual_seed(5)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = (torch.empty(3, h, 128, dtype=dt, device="cuda") for h in (8, 2, 2))
    out = [torch.empty_like(q) for _ in range(2)]

    def layers():
        for l in range(2):
            c.append(l, k, v)
            c.decode(l, q, out=out[l], prefix=prefix)
    graph = torch.cuda.CUDAGraph() if captured else None
    if captured:
        c.begin_step([False] * 3)                            # (kernels are loaded before they are captured)
        layers()
        c.cancel()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            layers()
        with pytest.raises(RuntimeError, match="prefix"):
            c.begin_step()
    for step in range(3):
        for x, h in ((q, 8), (k, 2), (v, 2)):
            x.copy_(random_rows(torch, g, dtype, 3, h, 128))
        c.begin_step(prefix=prefix)
        graph.replay() if captured else layers()
        c.advance()
        torch.cuda.synchronize()
        assert c.lens_host == [step + 1, 0, step + 1]
        for l in range(2):
            for s in (0, 2):
                K, V = (x.double().cpu().numpy() for x in c.read(l, s))
                for h in range(2):
                    parts = [unit_rows(prefix, raw, s, l, h, dtype), (K[h], V[h], np.zeros_like(K[h]), np.zeros_like(K[h]))]
                    want, bound = attend_parts(q[s, 4 * h:4 * h + 4].double().cpu().numpy(), parts, 1 / math.sqrt(128), dtype == "f32", False)
                    check(out[l][s, 4 * h:4 * h + 4].double().cpu().numpy(), want, bound, (step, l, s, h))
            assert (out[l][1] == 0).all()
