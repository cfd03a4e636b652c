"""Ties of fdkv_block_select: blocks whose bounds agree wherever the bound on the logits reads them
have one rank, and the lowest of them are selected."""
import pytest

from test_gpu_blocks import _same, _select, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,G,nb", [("f32", 128, 1, 300), ("f32", 64, 4, 5000), ("f32", 128, 8, 4096), ("bf16", 128, 4, 700)])
@pytest.mark.parametrize("signs", ["positive", "negative", "mixed"])
def test_equal_bounds_on_the_logits(torch_dev, dtype, d, G, nb, signs):
    """One value where a query reads it (the largest key under a positive channel, the least under a negative one),
    random ones on the other side: U is the same sum of the same products in every block."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] ties {dtype} d{d} G{G} {nb} blocks {signs}", flush=True)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(nb + d)
    sign = {"positive": torch.ones(d), "negative": -torch.ones(d), "mixed": 1 - 2 * (torch.rand(d, generator=g) < 0.5).float()}[signs]
    q = ((0.1 + torch.rand(1, 1, G, d, generator=g)) * sign).to(dt)
    read = torch.randn(d, generator=g)
    other = read - sign * 3 * torch.rand(1, 1, nb, d, generator=g)
    read = read.expand_as(other)
    bounds = torch.stack([torch.where(sign > 0, other, read), torch.where(sign > 0, read, other)], 3).to(dt)
    dims = B.dims(2, 1, G, d, 0, dtype)
    for first, last, n_sel in ((0, 0, 7), (2, 3, 200)):
        want = list(range(n_sel - last)) + list(range(nb - last, nb))
        _same(*_select(torch, B, dims, [nb * 64], bounds.cuda(), q.cuda(), first, last, n_sel), [want], n_sel)
