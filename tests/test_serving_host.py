"""Refusals of the serving entry points (rope, bounds, selection, parts) on the
host: every invalid call returns before any HIP call (the fake pointers are never
used), and the workspace queries."""
import ctypes
import os

import pytest

from paper_2607_06519_amd import binding as B

P = 1 << 20                     # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libfdkv.so not built")
    return B.load()


def _rope(rot=128, inter=0, axes=1, freq=P, pos=P, axis=()):
    return B.Rope(rot, inter, axes, freq, pos, (ctypes.c_uint8 * 64)(*axis))


def test_rope_append_refuses(lib):
    dm = B.dims(2, 2, 8, 128, 0, "bf16")

    def call(dims=dm, n=4, rope=_rope(), q=P, qs=1024, k=P, ks=256, v=P, vs=256, qn=None, kn=None, eps=1e-6, qo=2 * P,
             batch=2, seqs=None, rows=P, cap=8, ko=P, vo=P):
        return lib.fdkv_rope_append(ctypes.byref(dims) if dims else None, n, ctypes.byref(rope) if rope else None, q, qs, k, ks, v, vs, qn, kn,
                                    ctypes.c_float(eps), qo, batch, seqs, rows, cap, ko, vo, None)
    assert call(n=0) == 0
    assert call(dims=None) == -1 and call(rope=None) == -1 and call(n=-1) == -1
    assert call(batch=0) == -1 and call(cap=0) == -1
    for r in (_rope(rot=-16), _rope(rot=144), _rope(rot=24), _rope(inter=2), _rope(axes=0), _rope(axes=5), _rope(axis=[0, 1]),
              _rope(freq=0), _rope(pos=0), _rope(freq=P + 4), _rope(pos=P + 2)):
        assert call(rope=r) == -1
    assert call(dims=B.dims(2, 2, 8, 64, 0, "bf16"), rope=_rope(rot=128)) == -1
    for eps in (-1.0, float("nan"), float("inf")):
        assert call(qn=P, eps=eps) == -1 and call(kn=P, eps=eps) == -1
    for name in ("q", "k", "v", "qo", "ko", "vo", "rows"):
        assert call(**{name: None}) == -1 and call(**{name: P + 2}) == -1, name
    assert call(seqs=P + 1) == -1 and call(qn=P + 8) == -1 and call(kn=P + 8) == -1
    for name in ("qs", "ks", "vs"):
        assert call(**{name: -256}) == -1 and call(**{name: 260}) == -1 and call(**{name: 1 << 62}) == -1, name
    assert call(q=P, qo=P, qs=2048) == -1                       # in place only where the rows are contiguous
    assert call(dims=B.dims(2, 2, 6, 128, 0, "bf16")) == -2
    assert call(n=1 << 24) == -2 and call(n=2147483647) == -2


def test_key_bounds_refuses(lib):
    dm = B.dims(2, 2, 8, 128, 0, "bf16")
    good, bad = (ctypes.c_void_p * 2)(P, P), (ctypes.c_void_p * 2)(P, P + 8)
    call = lambda T=100, k=good, out=good, cap=2: lib.fdkv_key_bounds(ctypes.byref(dm), T, k, out, cap, None)
    assert call(T=0, cap=0) == 0
    assert call(T=-1) == -1 and call(k=None) == -1 and call(out=None) == -1 and call(cap=1) == -1
    assert call(k=bad) == -1 and call(out=bad) == -1
    assert call(T=2147483647, cap=1 << 26) == -2
    with pytest.raises(ValueError):
        B.key_bounds(dm, 100, [], [], 2)


def test_block_select_refuses(lib):
    dm = B.dims(2, 2, 8, 128, 0, "bf16")
    assert B.block_select_workspace(dm, 3, 1000) == 3 * 8 * 16 * 8
    assert B.block_select_workspace(dm, 1, 0) == 8 * 8

    def call(dims=dm, batch=3, lens=P, T=1000, bounds=P, q=P, first=1, last=2, sel=4, blocks=P, counts=P, ws=P, n=3 * 8 * 16 * 8):
        return lib.fdkv_block_select(ctypes.byref(dims), batch, lens, T, bounds, q, first, last, sel, blocks, counts, ws, n, None)
    assert call(n=3 * 8 * 16 * 8 - 1) == -3
    assert call(batch=0) == -1 and call(T=-1) == -1 and call(sel=0) == -1 and call(sel=2) == -1 and call(first=-1) == -1 and call(last=-1) == -1
    assert call(first=1 << 30, last=1 << 30, sel=4) == -1 and call(first=2147483647, last=2147483647, sel=2147483647) == -1
    for name, off in (("lens", 2), ("bounds", 8), ("q", 8), ("blocks", 2), ("counts", 1), ("ws", 4)):
        assert call(**{name: None}) == -1 and call(**{name: P + off}) == -1, name
    assert call(batch=32768, n=1 << 62) == -2
    assert call(T=2147483647, n=1 << 62) == -2 and call(sel=(1 << 24) + 1) == -2 and call(sel=2147483647) == -2


def _part(kind=0, T=100, n_sel=0, lens=P, modes=P, offs=P, cache=P, blocks=None, counts=None):
    return B.Part(kind, T, n_sel, lens, modes, offs, cache, blocks, counts)


def test_decode_parts_refuses(lib):
    dm = B.dims(2, 2, 8, 128, 16, "bf16")
    tail = B.Tail(P, 8, P, P)

    def call(parts=(_part(),), tail=tail, batch=2, layer=0, q=P, out=P, scale=0.1, ws=P, n=1 << 40, dims=dm, count=None):
        arr = (B.Part * max(len(parts), 1))(*parts) if parts is not None else None
        return lib.fdkv_decode_parts(ctypes.byref(dims), batch, len(parts) if count is None else count, arr, ctypes.byref(tail) if tail else None,
                                     layer, q, out, ctypes.c_float(scale), ws, n, None)
    need = B.decode_parts_workspace(dm, 2, [_part()], 8)
    assert call(n=need - 1) == -3
    assert call(batch=0) == -1 and call(layer=-1) == -1 and call(layer=2) == -1 and call(count=-1) == -1 and call(parts=None, count=1) == -1
    assert call(parts=[_part()] * 16) == -1 and call(parts=[_part()] * 17, tail=None) == -1
    for name in ("q", "out", "ws"):
        assert call(**{name: None}) == -1 and call(**{name: P + 8}) == -1, name
    assert call(scale=float("nan")) == -1
    for p in (_part(kind=3), _part(kind=-1), _part(T=-1), _part(kind=1), _part(kind=1, n_sel=4), _part(kind=1, n_sel=4, blocks=P),
              _part(kind=1, n_sel=4, blocks=P + 2, counts=P), _part(lens=None), _part(lens=P + 2), _part(modes=P + 1), _part(offs=P + 4),
              _part(cache=P + 128), _part(cache=None), _part(kind=2, cache=None)):
        assert call(parts=[p]) == -1, list(getattr(p, f[0]) for f in p._fields_)
    assert call(parts=[_part(T=1 << 23)]) == -2 and call(parts=[_part(kind=2, T=1 << 23)]) == -2
    assert call(tail=B.Tail(P, 1 << 23, P, P)) == -2
    for t in (B.Tail(P, -1, P, P), B.Tail(P + 2, 8, P, P), B.Tail(P, 8, None, P), B.Tail(P, 8, P, P + 8)):
        assert call(tail=t) == -1
    tok = B.dims(4, 2, 8, 128, 0, "bf16", B.QUADS, B.RES_TOKENS, 1000000)
    assert call(dims=tok, parts=[_part(T=3000000)]) == -2        # rows of a set past 32-bit offsets
    n = ctypes.c_size_t(0)
    assert lib.fdkv_decode_parts_workspace(ctypes.byref(dm), 2, 0, None, -1, ctypes.byref(n)) == 0 and n.value == 2 * 2 * 4 * 132 * 4
    assert lib.fdkv_decode_parts_workspace(ctypes.byref(dm), 2, 0, None, -1, None) == -1
    for batch in ((1 << 20) + 1, 1 << 30, 2147483647):
        assert lib.fdkv_decode_parts_workspace(ctypes.byref(dm), batch, 0, None, -1, ctypes.byref(n)) == -2
    assert call(parts=[_part(kind=1, n_sel=(1 << 24) + 1, blocks=P, counts=P)]) == -2
    assert call(parts=[_part(T=1 << 22)], batch=1 << 18) == -2   # more record slots than a launch has workgroups


def test_parts_workspace(lib):
    """Records of every part's slots, a slot at least per 64 tokens of the bound (a shared part: or as many as one
    residual head among plain ones may take), and never less for a longer bound at the same split."""
    for dtype in ("bf16", "f32", "bf16_e4m3"):
        dm = B.dims(2, 8, 32, 128, 16, dtype)
        rec = 4 * 132 * 4
        for batch in (1, 16, 200):
            for kind in (0, 2):
                for T in (0, 1, 32, 33, 5000, 131072):
                    n = B.decode_parts_workspace(dm, batch, [_part(kind, T)], -1)
                    slots = n // (batch * 8 * rec)
                    assert 1 <= slots <= max(1, -(-T // 64)) * (3 if kind == 2 else 1) + 1
                    assert n - slots * batch * 8 * rec in (0, 256)
