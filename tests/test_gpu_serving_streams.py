"""The serving step's operators on a stream that is not the current one: what a call allocates
is neither in use by the current stream nor written by it afterwards."""
import pytest

from serving_cases import make_cache
from test_gpu_parts import _dims, _modes, log, torch_dev  # noqa: F401
from test_gpu_serving_step import EPS, Step

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


@pytest.mark.parametrize("shared", [300, 0])
def test_outputs_of_a_side_stream(torch_dev, shared):
    """A step on a side stream, its outputs allocated by the calls, while the current stream still has to read what
    was freed there: that is not overwritten, and the outputs are those of a step on the current stream."""
    torch = torch_dev
    st = Step(torch, "bf16", shared=shared, lens=(1000, 64, 517), select=(1, 1, 4) if shared else None)
    st.new_inputs(40)
    st.run()
    want_q, want = [t.clone() for t in st.q], [t.clone() for t in st.out]
    dm, gen, side = st.dims, st.gen, torch.cuda.Stream()
    plain = st.prefix.decode(0, want_q[0])
    log(f"[case] outputs beside a busy stream, shared {shared}")
    old = [torch.full_like(want[0], 7.0) for _ in range(12)]
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    kept = [t.clone() for t in old]
    del old
    got = []
    for l in range(dm.n_layers):
        q, k, v = st.rows[l].split((dm.n_q_heads, dm.n_kv_heads, dm.n_kv_heads), 1)
        q = gen.append_rotated(l, st.rope, q, k, v, *st.norm, eps=EPS, stream=side)
        got.append((q, gen.decode(l, q, stream=side)))
    got_plain = st.prefix.decode(0, want_q[0], stream=side)
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in kept)
    for l, (q, out) in enumerate(got):
        assert torch.equal(q, want_q[l]) and torch.equal(out, want[l]), l
    assert torch.equal(got_plain, plain)


def test_append_rotated_into_given_queries(torch_dev):
    torch = torch_dev
    st = Step(torch, "bf16")
    st.new_inputs(3)
    st.run()
    dm = st.dims
    q, k, v = st.rows[1].split((dm.n_q_heads, dm.n_kv_heads, dm.n_kv_heads), 1)
    out = torch.zeros_like(st.q[1])
    assert st.gen.append_rotated(1, st.rope, q, k, v, *st.norm, eps=EPS, out=out) is out and torch.equal(out, st.q[1])
    for bad in (out.float(), out[:, :-1], out[:, :, ::2]):
        with pytest.raises(ValueError):
            st.gen.append_rotated(1, st.rope, q, k, v, out=bad)
