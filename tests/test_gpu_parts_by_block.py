"""fdkv_decode_parts within the bound of the very block that a layer is of: pairs, whose residual is a stored
value and goes in exactly, have nothing of what serving_cases grants the weighted sums of a block of four."""
import numpy as np
import pytest

import test_gpu_parts as parts
from test_gpu_parts import KINDS, Case, _kind, log, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu

PAIRS = [name for name, kind in KINDS.items() if kind[4] != 2]


@pytest.fixture(autouse=True)
def by_block(monkeypatch):
    """Case.want with the bound of its layer's block."""
    want, attend = Case.want, parts.attend

    def of_layer(self, layer):
        from paper_2607_06519_amd import binding as B
        first, size = B.blocks(self.dims)
        quads = any(f <= layer < f + n and n == 4 for f, n in zip(first, size))
        monkeypatch.setattr(parts, "attend", lambda q, p, scale, f32, _: attend(q, p, scale, f32, quads))
        return want(self, layer)
    monkeypatch.setattr(Case, "want", of_layer)


@pytest.mark.parametrize("name", PAIRS)
def test_shared_and_own(torch_dev, name):
    dims, dtype, layers = _kind(name)
    G = dims.n_q_heads // dims.n_kv_heads
    log(f"[case] by block {name}")
    for batch in (3, 40 // G + 1, 120 // G + 1):
        Case(torch_dev, dims, dtype, batch, 1100 + batch, shared=(219,), own=([(53 * s) % 150 for s in range(batch)],),
             tail=(9, [s % 10 for s in range(batch)])).check(layers, f"{name} b{batch}")


@pytest.mark.parametrize("name", PAIRS)
def test_blocks(torch_dev, name):
    dims, dtype, layers = _kind(name)
    rng = np.random.default_rng(4)
    lens = [517, 64, 0, 1000]
    lists = [[sorted(rng.permutation(-(-T // 64))[:rng.integers(0, 7)].tolist()) for _ in range(dims.n_kv_heads)] for T in lens]
    log(f"[case] by block, selected {name}")
    Case(torch_dev, dims, dtype, 4, 1200, blocks=(lens, lists, 9), tail=(70, [3, 70, 1, 33])).check(layers, name)
