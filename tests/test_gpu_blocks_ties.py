"""Ties of fdkv_block_select: blocks whose bounds agree wherever the bound on the logits reads them
have one rank, and the lowest of them are selected."""
import numpy as np
import pytest

from test_gpu_blocks import _same, _select, _want, torch_dev  # noqa: F401

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


def _bounds(kind, nb, d, rng):
    """Bounds [1][1][nb][2][d] and queries [1][1][2][d] whose ranks tie, spread or bunch."""
    x = np.zeros((1, 1, nb, 2, d), np.float32)
    q = np.zeros((1, 1, 2, d), np.float32)
    q[..., 0, 0] = q[..., 1, 1] = 1
    if kind == "zero_query":
        q[:] = 0
        x[:] = rng.standard_normal(x.shape)
    elif kind == "equal":
        x[:] = 1
    elif kind == "two_values":
        x[0, 0, :, :, 0] = -1.0 * (rng.integers(0, 10, (nb, 1)) > 0)
        x[0, 0, :, :, 1] = -9
    elif kind == "steps":
        x[0, 0, :, :, 0] = -rng.integers(0, 3, (nb, 1)) / 4096   # three ranks, in one bin beside an outlier
        x[0, 0, nb // 2, :, 0] = -1e6
        x[0, 0, :, :, 1] = -2e6
    elif kind == "huge":
        x[0, 0, :, :, 0] = -np.exp2(rng.integers(-60, 100, (nb, 1)))
        x[0, 0, :, :, 1] = -3e38
    else:
        x[0, 0, :, :, 0] = -1 + 1e-6 * rng.random((nb, 1))       # distinct, in one bin
        x[0, 0, 77, :, 0] = 0
        x[0, 0, 78, :, 0] = -1e30
        x[0, 0, :, :, 1] = -1e35
    return np.sort(x, 3), q


@pytest.mark.parametrize("nb", [513, 600, 4096, 4097])
@pytest.mark.parametrize("kind", ["zero_query", "equal", "two_values", "steps", "huge", "one_apart"])
def test_ties_where_the_ranks_are_held(torch_dev, kind, nb):
    """Up to 4096 blocks a workgroup keeps the ranks in LDS: more equal ranks, or ranks in one bin, than its list takes,
    on both sides of that."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    print(f"[case] {kind} of {nb} blocks", flush=True)
    x, q = _bounds(kind, nb, 64, np.random.default_rng(nb))
    dims = B.dims(2, 1, 2, 64, 0, "f32")
    for first, last, n_sel in ((0, 0, 100), (1, 3, 100), (2, 0, 512), (0, 0, 1)):
        want = _want(x.astype(np.float64), q.astype(np.float64), [nb * 64], first, last, n_sel)
        _same(*_select(torch, B, dims, [nb * 64], torch.from_numpy(x).cuda(), torch.from_numpy(q).cuda(), first, last, n_sel), want, n_sel)
