"""CompressedCache and Generation around the serving step, on the host: which calls they refuse.  The
library's device calls are replaced by stubs; everything else is their own code on CPU tensors."""
import os

import numpy as np
import pytest

from paper_2607_06519_amd import binding as B
from paper_2607_06519_amd import cache as C


@pytest.fixture
def calls(monkeypatch):
    import torch
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libfdkv.so not built")
    seen = []
    monkeypatch.setattr(C, "_torch", lambda: torch)
    for name in ("compress", "key_bounds", "block_select", "decode_parts"):
        monkeypatch.setattr(C.B, name, lambda *a, _name=name, **k: seen.append(_name))
    return seen


DIMS = B.dims(2, 2, 8, 128, 16, "bf16")


def _cache(lens, dims=DIMS):
    return C.CompressedCache(dims, lens, np.zeros((len(lens), len(B.blocks(dims)[0]), dims.n_kv_heads), np.uint8), device="cpu")


def _sparse(prefix, select=(1, 1, 4)):
    return C.Generation(DIMS, prefix, 4, device="cpu", select=select)


def test_a_sequence_compressed_again_is_indexed_again(calls):
    import torch
    q = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    c = _cache([200, 100])
    for s in range(2):
        c.compress(s, [], [])
        c.index(s, [])
    gen = _sparse(c)
    gen.decode(0, q)
    c.compress(1, [], [])                                    # other keys
    calls.clear()
    with pytest.raises(RuntimeError):
        gen.decode(0, q)
    assert not calls
    with pytest.raises(ValueError):
        _sparse(c)
    c.index(1, [])
    gen.decode(0, q)
    _sparse(c)


def test_indexed_before_or_after_the_first_compression(calls):
    c = _cache([200, 0, 100])
    c.index(0, [])
    c.compress(0, [], [])
    c.compress(2, [], [])
    c.index(2, [])
    c.compress(1, [], [])
    c.compress(1, [], [])                                    # an empty sequence has no bounds
    _sparse(c)


def test_a_selection_that_the_library_refuses_is_refused_at_once(calls):
    c = _cache([200, 100])
    for s in range(2):
        c.index(s, [])
    for select in ((0, 0, 1), (2, 2, 4), (0, 0, 1 << 12)):
        assert _sparse(c, select).select == select
    for select in ((3, 3, 4), (0, 0, 0), (-1, 0, 4), (0, -1, 4), (0, 0, -4), (0, 0, (1 << 24) + 1)):
        with pytest.raises(B.FdkvError):
            _sparse(c, select)
    for select in ((1, 4), (1, 1, 4, 4)):
        with pytest.raises(ValueError):
            _sparse(c, select)


def test_a_prefix_of_empty_sequences(calls):
    """Nothing to index, and nothing to select from: the bounds are there all the same, for their address."""
    import torch
    gen = _sparse(_cache([0, 0]))
    gen.decode(0, torch.zeros(2, 8, 128, dtype=torch.bfloat16))
    assert calls == ["block_select", "decode_parts"] and all(b.data_ptr() for b in gen.spans[0].bounds)


@pytest.mark.parametrize("which", ["shared", "beside", "sparse"])
def test_a_prefix_of_another_cache(calls, which):
    def make(dims):
        if which == "shared":
            return C.Generation(DIMS, None, 4, device="cpu", shared=_cache([200], dims), batch=2)
        if which == "beside":
            return C.Generation(DIMS, _cache([200, 0], dims), 4, device="cpu", shared=_cache([100]))
        return C.Generation(DIMS, _cache([0, 0], dims), 4, device="cpu", select=(0, 0, 1))
    make(DIMS)
    make(B.dims(2, 2, 4, 128, 16, "bf16"))                   # (the query heads are not the cache's)
    for dims in (B.dims(4, 2, 8, 128, 16, "bf16"), B.dims(2, 4, 8, 128, 16, "bf16"), B.dims(2, 2, 8, 64, 16, "bf16"),
                 B.dims(2, 2, 8, 128, 8, "bf16"), B.dims(2, 2, 8, 128, 16, "bf16_e4m3"), B.dims(2, 2, 8, 128, 16, "f32"),
                 B.dims(2, 2, 8, 128, 16, "bf16", residual=B.RES_TOKENS, res_ppm=10000)):
        with pytest.raises(ValueError):
            make(dims)
