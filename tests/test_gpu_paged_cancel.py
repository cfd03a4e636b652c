"""PagedCache: prompts and steps that are given up on their way, and made again."""
import pytest

from rows_cases import random_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from paper_2607_06519_amd import binding
    binding.load()
    return torch


@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3", "f32"])
def test_made_again(torch_dev, dtype):
    """A piece and a step that fail, are cancelled and are made again give the bits of those that do not fail; rows of what
    was cancelled are of no sequence."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    from paper_2607_06519_amd.cache import PagedCache
    print(f"[case] cancel {dtype}", flush=True)
    dims = B.dims(2, 2, 8, 128, 0, dtype)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(3)
    rows_of = lambda n: [random_rows(torch, g, dtype, n, h, 128).to(dt).cuda() for h in (8, 2, 2)]
    pieces = [([20, 33], rows_of(53)), ([50, 7], rows_of(57))]
    step = rows_of(2)
    held, outs = [], []
    for fail in (False, True):
        c = PagedCache(dims, 2, 100, page=16)
        given = []
        for counts, (q, k, v) in pieces:
            if fail:
                rows = c.begin(counts)
                c.prompt(rows, 0, -q, -2 * k, -2 * v)
                with pytest.raises(ValueError):
                    c.prompt(rows, 1, q, k, v[1:])
                c.cancel()
            rows = c.begin(counts)
            given += [c.prompt(rows, l, q, k, v) for l in range(2)]
            c.end(rows)
        if fail:
            c.begin_step()
            c.append(0, -step[1], -step[2])
            with pytest.raises(ValueError):
                c.append(1, step[1][1:], step[2])
            c.cancel()
            c.end(c.begin([0, 0]))
        c.begin_step()
        for l in range(2):
            c.append(l, step[1], step[2])
            given.append(c.decode(l, step[0]))
        c.advance()
        held.append([x for l in range(2) for s in range(2) for x in c.read(l, s)])
        outs.append(given)
    torch.cuda.synchronize()
    assert c.lens_host == [71, 41]
    assert all(torch.equal(a, b) for a, b in zip(outs[0] + held[0], outs[1] + held[1]))
