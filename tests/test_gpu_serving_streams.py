"""The serving step's operators on a stream that is not the current one: what a call allocates
is neither in use by the current stream nor written by it afterwards."""
import pytest

from serving_cases import make_cache
from test_gpu_parts import _dims, _modes, log, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu

BUSY = 20_000_000  # clock cycles that keep the current stream occupied: some 10 ms


def _bounds(torch, k):
    return torch.stack([torch.stack([x.amin(1), x.amax(1)], 1) for x in k.split(64, 1)], 1)


def test_first_index_on_a_side_stream(torch_dev):
    """The current stream is busy while another one writes the first bounds: they are kept, and what the current
    stream still reads of the memory that they take is not overwritten."""
    torch = torch_dev
    dims = _dims("bf16", 2, 4, 128, 16)
    cache, keys = make_cache(torch, dims, [700, 130], _modes(dims, 2, 4), 960)
    side = torch.cuda.Stream()
    log("[case] index beside a busy stream")
    old = [torch.full((2, 2, 11, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(dims.n_layers)]
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    kept = [t.clone() for t in old]
    del old
    for s in range(2):
        cache.index(s, keys[s], stream=side)
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in kept)
    for l in range(dims.n_layers):
        for s, T in enumerate((700, 130)):
            assert torch.equal(cache.bounds[l][s, :, :-(-T // 64)], _bounds(torch, keys[s][l])), (l, s)
