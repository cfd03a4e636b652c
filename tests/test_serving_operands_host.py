"""Operands that a kernel of the serving step would read past their end, or on another device than its own, are
refused before any call of the library (the tensors here are on the CPU, and no kernel runs)."""
import os

import pytest

from paper_2607_06519_amd import binding as B


@pytest.fixture
def cpu(monkeypatch):
    """CPU tensors pass for the current device's; a call that is not refused ends in Queued."""
    import torch
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libfdkv.so not built")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)

    class Queued(Exception):
        pass

    def queued(*a):
        raise Queued
    monkeypatch.setattr(B, "_stream", queued)
    torch.Queued = Queued
    yield torch
    del torch.Queued


BATCH, NSEL = 3, 5


def _part(torch, kind, dims, seqs, n_sel=0, short=None):
    """A part of ``seqs`` sequences whose ``short`` operand is one value short."""
    units = dims.n_kv_heads * B._n_blocks(dims.n_layers, dims.schedule)
    n = dict(seq_lens=seqs, modes=seqs * units, seg_offsets=seqs * units, blocks=seqs * dims.n_kv_heads * n_sel, counts=seqs * dims.n_kv_heads)
    types = dict(seq_lens=torch.int32, modes=torch.uint8, seg_offsets=torch.int64, blocks=torch.int32, counts=torch.int32)
    t = {k: torch.zeros(m - (k == short), dtype=types[k]) for k, m in n.items()}
    if kind != B.PART_BLOCKS:
        t["blocks"] = t["counts"] = None
    return B.part(kind, t["seq_lens"], 100, t["modes"], t["seg_offsets"], torch.zeros(256, dtype=torch.uint8), t["blocks"], t["counts"], n_sel)


@pytest.mark.parametrize("schedule,layers", [(0, 4), (1, 12), (2, 4)])
def test_parts_shorter_than_the_batch(cpu, schedule, layers):
    torch = cpu
    dims = B.dims(layers, 2, 8, 128, 16, "bf16", schedule)
    q = torch.zeros(BATCH, 8, 128, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 20)
    call = lambda *parts, ws=ws: B.decode_parts(dims, BATCH, parts, None, 0, q, torch.zeros_like(q), 0.1, ws)
    kinds = ((B.PART_OWN, BATCH, 0), (B.PART_SHARED, 1, 0), (B.PART_BLOCKS, BATCH, NSEL))
    for kind, seqs, n_sel in kinds:
        good = _part(torch, kind, dims, seqs, n_sel)
        with pytest.raises(torch.Queued):
            call(good)
        for short in ("seq_lens", "modes", "seg_offsets") + (("blocks", "counts") if n_sel else ()):
            with pytest.raises(ValueError):
                call(good, _part(torch, kind, dims, seqs, n_sel, short))
        if kind != B.PART_SHARED:
            with pytest.raises(ValueError):
                call(_part(torch, kind, dims, BATCH - 1, n_sel))
    grown = _part(torch, B.PART_BLOCKS, dims, BATCH, NSEL)
    with pytest.raises(torch.Queued):
        call(grown)
    more = torch.zeros(BATCH + 1, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):                              # the same descriptor in a call for more
        B.decode_parts(dims, BATCH + 1, [grown], None, 0, more, torch.zeros_like(more), 0.1, ws)
    grown.n_sel = NSEL + 1
    with pytest.raises(ValueError):
        call(grown)


def test_workspaces_on_another_device(cpu):
    torch = cpu

    class Elsewhere:                                             # what a tensor of another device says of itself
        device, get_device, is_contiguous, stride = "cuda:7", lambda s: 7, lambda s: True, lambda s: (1,)
        numel, element_size, data_ptr = lambda s: 1 << 20, lambda s: 4, lambda s: 1 << 20
    dims = B.dims(2, 2, 8, 128, 16, "bf16")
    q = torch.zeros(BATCH, 8, 128, dtype=torch.bfloat16)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    bounds = torch.zeros(BATCH, 2, 16, 2, 128, dtype=torch.bfloat16)
    for ws in (Elsewhere(), torch.zeros(1 << 20)[::2]):
        with pytest.raises(ValueError):
            B.decode_parts(dims, BATCH, [_part(torch, B.PART_OWN, dims, BATCH)], None, 0, q, torch.zeros_like(q), 0.1, ws)
        with pytest.raises(ValueError):
            B.block_select(dims, BATCH, i32(BATCH), 1000, bounds, q, 0, 1, 4, i32(BATCH, 2, 4), i32(BATCH, 2), ws)
    with pytest.raises(torch.Queued):
        B.block_select(dims, BATCH, i32(BATCH), 1000, bounds, q, 0, 1, 4, i32(BATCH, 2, 4), i32(BATCH, 2), torch.zeros(1 << 20))


def test_axes_of_pairs():
    import torch
    freq = torch.zeros(8, dtype=torch.float64)
    pos = torch.zeros(2, 3, dtype=torch.int32)
    assert B.rope(16, freq, pos, [0, 1] * 4).axis[1] == 1
    for axis in ([0, 2] * 4, [0, 256] * 4, [-1, 0] * 4, [0, 1] * 3):   # (256 is 0 in eight bits)
        with pytest.raises(ValueError):
            B.rope(16, freq, pos, axis)
