"""Refusals of the entry points of exact rows (prompt attention, pages, decode over pages) on the host: every invalid call
returns before any HIP call (the fake pointers are never used), the workspace queries, and operands that a kernel would
misread (the tensors here are on the CPU, and no kernel runs)."""
import ctypes
import os

import pytest

from paper_2607_06519_amd import binding as B

P = 1 << 20                     # an aligned address that nothing reads
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libfdkv.so not built")
    return B.load()


def test_prompt_attn_refuses(lib):
    dm = B.dims(2, 2, 8, 128, 0, "bf16")
    need = B.prompt_attn_workspace(dm, 4, 2, 4000)
    assert need > 0 and B.prompt_attn_workspace(dm, 100000, 2, 4000) == 0 and B.prompt_attn_workspace(dm, 0, 1, 0) == 0

    def call(dims=dm, n=4, q=P, qs=1024, batch=2, starts=P, k=P, ks=(0, 128, 256), v=P, vs=(0, 128, 256), rows=4000, first=None, lens=P,
             out=2 * P, scale=0.1, ws=P, size=need):
        s3 = lambda s: (ctypes.c_int64 * 3)(*s) if s else None
        return lib.fdkv_prompt_attn(ctypes.byref(dims) if dims else None, n, q, qs, batch, starts, k, s3(ks), v, s3(vs), rows, first, lens, out,
                                    ctypes.c_float(scale), ws, size, None)
    assert call(n=0) == 0
    assert call(size=need - 1) == -3 and call(ws=None) == -1 and call(ws=P + 4) == -1
    assert call(dims=None) == -1 and call(n=-1) == -1 and call(batch=0) == -1 and call(rows=-1) == -1
    for name, off in (("q", 8), ("starts", 2), ("k", 8), ("v", 8), ("lens", 2), ("out", 8)):
        assert call(**{name: None}) == -1 and call(**{name: P + off}) == -1, name
    assert call(rows=0, k=P + 8, n=0) == 0
    assert call(first=P + 2) == -1 and call(scale=NAN) == -1 and call(scale=INF) == -1
    assert call(qs=-128) == -1 and call(qs=129) == -1 and call(qs=1 << 62) == -1
    for name in ("ks", "vs"):
        assert call(**{name: None}) == -1
        for i in range(3):
            for bad in (-128, 129, 1 << 62):
                s = [0, 128, 256]
                s[i] = bad
                assert call(**{name: s}) == -1, (name, i, bad)
        assert call(**{name: (0, 128, 1 << 23)}) == -2
    assert call(q=P, out=P, qs=2048) == -1                       # in place only where the rows are contiguous
    assert call(n=1 << 24) == -2 and call(n=2147483647) == -2 and call(batch=65536) == -2
    assert call(dims=B.dims(2, 2, 6, 128, 0, "bf16")) == -2
    assert call(dims=B.dims(2, 4096, 4096, 128, 0, "bf16"), n=(1 << 24) - 1) == -2
    n = ctypes.c_size_t(0)
    assert lib.fdkv_prompt_attn_workspace(ctypes.byref(dm), 4, 2, 4000, None) == -1
    assert lib.fdkv_prompt_attn_workspace(ctypes.byref(dm), -1, 2, 4000, ctypes.byref(n)) == -1


def test_prompt_workspace(lib):
    """Records of every query row and split, and none where the rows alone fill the card."""
    for dtype in ("bf16", "f32"):
        for d, G in ((64, 1), (128, 4), (128, 8)):
            dm = B.dims(2, 8, 8 * G, d, 0, dtype)
            least = 64 if dtype == "f32" else 1024
            for n in (1, 7, 250, 3000):
                for batch in (1, 5):
                    for rows in (0, 1, 256, 257, 5000, 1 << 20, 2147483647):
                        size = B.prompt_attn_workspace(dm, n, batch, rows)
                        record = n * 8 * G * (d + 4) * 4
                        assert size % record == 0 and size // record in (0, *range(2, 513)), (n, batch, rows)
                        assert rows > least or size == 0


def _pages(n_pages=4, page=16, batch=2, most=3, table=P, k=P, v=P, ke=P, ve=P):
    return B.Pages(n_pages, page, batch, most, table, k, v, ke, ve)


BAD = [_pages(n_pages=0), _pages(batch=0), _pages(most=0), _pages(table=None), _pages(table=P + 2), _pages(k=None), _pages(v=P + 8)] + \
      [_pages(page=p) for p in (0, -16, 1, 8, 15, 17, 48, 512, 1 << 30)]
BAD8 = [_pages(ke=None), _pages(ve=None), _pages(ke=P + 8), _pages(ve=P + 4)]


def test_page_rows_refuse(lib):
    for f in (lib.fdkv_page_write, lib.fdkv_page_read):
        for dtype in ("bf16", "bf16_e4m3", "f32"):
            dm = B.dims(2, 2, 8, 128, 0, dtype)

            def call(pg=_pages(), n=4, k=P, ks=(256, 128), v=P, vs=(256, 128), seqs=None, rows=P, dims=dm):
                s2 = lambda s: (ctypes.c_int64 * 2)(*s) if s else None
                return f(ctypes.byref(dims), ctypes.byref(pg) if pg else None, n, k, s2(ks), v, s2(vs), seqs, rows, None)
            assert call(n=0) == 0 and call(pg=None) == -1 and call(n=-1) == -1 and call(n=(1 << 24) + 1) == -2 and call(n=2147483647) == -2
            for pg in BAD + (BAD8 if dtype == "bf16_e4m3" else []):
                assert call(pg=pg) == -1
            for name, off in (("k", 8), ("v", 8), ("rows", 2)):
                assert call(**{name: None}) == -1 and call(**{name: P + off}) == -1, name
            assert call(seqs=P + 2) == -1
            for name in ("ks", "vs"):
                assert call(**{name: None}) == -1
                for bad in ((-128, 128), (256, -8), (257, 128), (256, 1 << 62)):
                    assert call(**{name: bad}) == -1, bad
            assert call(dims=B.dims(2, 1 << 22, 1 << 22, 128, 0, dtype), n=9) == -2


def test_paged_attn_refuses(lib):
    for dtype in ("bf16", "bf16_e4m3", "f32"):
        dm = B.dims(2, 2, 8, 128, 0, dtype)
        need = B.paged_attn_workspace(dm, 2, 48)
        assert need == 2 * 2 * 4 * 132 * 4

        def call(pg=_pages(), lens=P, most=48, more=None, n_more=0, q=P, out=P, scale=0.1, ws=P, size=need):
            return lib.fdkv_paged_attn(ctypes.byref(dm), ctypes.byref(pg) if pg else None, lens, most, more, n_more, q, out,
                                       ctypes.c_float(scale), ws, size, None)
        assert call(size=need - 1) == -3 and call(pg=None) == -1
        for pg in BAD + (BAD8 if dtype == "bf16_e4m3" else []):
            assert call(pg=pg) == -1
        assert call(most=-1) == -1 and call(most=49) == -1 and call(n_more=-1) == -1 and call(n_more=1) == -1 and call(more=P + 8, n_more=1) == -1
        assert call(more=P, n_more=(1 << 20) + 1) == -2
        for name, off in (("lens", 2), ("q", 8), ("out", 8), ("ws", 8)):
            assert call(**{name: None}) == -1 and call(**{name: P + off}) == -1, name
        assert call(scale=NAN) == -1
        assert call(pg=_pages(page=256, most=1 << 23), most=(1 << 30) + 1) == -2
        n = ctypes.c_size_t(0)
        assert lib.fdkv_paged_attn_workspace(ctypes.byref(dm), 0, 1, ctypes.byref(n)) == -1
        assert lib.fdkv_paged_attn_workspace(ctypes.byref(dm), 1, -1, ctypes.byref(n)) == -1
        assert lib.fdkv_paged_attn_workspace(ctypes.byref(dm), 1, 1, None) == -1
        assert lib.fdkv_paged_attn_workspace(ctypes.byref(dm), 1 << 22, 1, ctypes.byref(n)) == -2
        assert lib.fdkv_paged_attn_workspace(ctypes.byref(dm), 1 << 14, 1 << 20, ctypes.byref(n)) == -2
        assert lib.fdkv_paged_attn_workspace(ctypes.byref(dm), 2147483647, 1 << 30, ctypes.byref(n)) == -2


def test_paged_workspace_serves_shorter_calls(lib):
    """The query never gives less for more tokens, nor less than a call's chunks of at least 128 tokens need."""
    for batch, kv in ((1, 1), (1, 8), (3, 2), (64, 8), (300, 1)):
        dm = B.dims(2, kv, 4 * kv, 128, 0, "bf16")
        last, unit = 0, batch * kv * 4 * 132 * 4
        for m in sorted({*range(0, 3000, 97), *range(32500, 33100), *(1 << i for i in range(21)), *((1 << i) + 1 for i in range(21))}):
            n = B.paged_attn_workspace(dm, batch, m)
            assert n >= last and unit <= n <= unit * max(1, -(-m // 128)), (batch, kv, m)
            last = n


@pytest.fixture
def cpu(monkeypatch, lib):
    """CPU tensors pass for the current device's; a call that is not refused ends in Queued."""
    import torch

    class Queued(Exception):
        pass

    def queued(*a):
        raise Queued
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", queued, raising=False)
    torch.Queued = Queued
    yield torch
    del torch.Queued


def test_prompt_operands(cpu):
    torch = cpu
    dims = B.dims(2, 2, 8, 128, 0, "bf16")
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    good = dict(q=z(5, 8, 128), k=z(3, 2, 9, 128), v=z(3, 2, 9, 128), q_starts=i32(4), k_lens=i32(3), out=z(5, 8, 128), ws=z(1 << 16, dt=torch.float32),
                k_starts=i32(3))
    call = lambda **o: B.prompt_attn(dims, sm_scale=0.1, **{**good, **o})
    for o in ({}, dict(k_starts=None), dict(k=z(1, 2, 9, 128), v=z(1, 2, 9, 128)), dict(q=z(5, 10, 128)[:, 1:9]),
              dict(k=z(9, 5, 128)[:, :2].transpose(0, 1)[None], v=z(9, 5, 128)[:, 2:4].transpose(0, 1)[None])):
        with pytest.raises(torch.Queued):
            call(**o)
    bad = [dict(q=z(5, 4, 128)), dict(q=z(5, 8, 64)), dict(q=z(8, 5, 128).transpose(0, 1)), dict(q=z(5, 8, 128, dt=torch.float32)),
           dict(out=z(4, 8, 128)), dict(out=z(8, 5, 128).transpose(0, 1)), dict(k=z(2, 2, 9, 128), v=z(2, 2, 9, 128)), dict(v=z(3, 2, 8, 128)),
           dict(k=z(3, 2, 9, 256)[..., ::2]), dict(k=z(3, 2, 9, 128, dt=torch.float16)), dict(q_starts=i32(3)), dict(q_starts=torch.zeros(4, dtype=torch.int64)),
           dict(k_starts=i32(2)), dict(k_lens=i32(6)[::2]), dict(ws=z(1 << 16, dt=torch.float32)[::2])]
    for o in bad:
        with pytest.raises(ValueError):
            call(**o)


def test_page_operands(cpu):
    torch = cpu
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)
    u8 = lambda *n: torch.zeros(*n, dtype=torch.uint8)
    dims, dims8 = B.dims(2, 2, 8, 128, 0, "bf16"), B.dims(2, 2, 8, 128, 0, "bf16_e4m3")
    pg = B.pages(dims, z(4, 2, 16, 128), z(4, 2, 16, 128), i32(3, 2))
    pg8 = B.pages(dims8, u8(4, 2, 16, 128), z(4, 2, 16, 128, dt=torch.float8_e4m3fn), i32(3, 2), u8(4, 2, 16), u8(4, 2, 16))
    k = z(4, 2, 16, 128)
    for d, a in ((dims, (k, z(4, 2, 8, 128), i32(3, 2))), (dims, (k, k, i32(6))), (dims, (k, k, i32(3, 2), u8(4, 2, 16), u8(4, 2, 16))),
                 (dims8, (u8(4, 2, 16, 128), u8(4, 2, 16, 128), i32(3, 2))), (dims8, (u8(4, 2, 16, 128), u8(4, 2, 16, 128), i32(3, 2), u8(4, 2, 16), u8(4, 2, 8))),
                 (dims8, (k, k, i32(3, 2), u8(4, 2, 16), u8(4, 2, 16))), (dims, (u8(4, 2, 16, 128), k, i32(3, 2))), (dims, (k, k, torch.zeros(3, 2))),
                 (dims, (z(4, 2, 128, 16).transpose(2, 3), k, i32(3, 2))), (dims, (k, k, i32(2, 3).T)), (dims, (z(4, 16, 2, 128), z(4, 16, 2, 128), i32(3, 2))),
                 (dims, (z(4, 2, 24, 128), z(4, 2, 24, 128), i32(3, 2))), (dims, (z(4, 2, 512, 128), z(4, 2, 512, 128), i32(3, 2)))):
        with pytest.raises(ValueError):
            B.pages(d, *a)
    rows = z(5, 2, 128)
    for f, d, p in ((f, d, p) for f in (B.page_write, B.page_read) for d, p in ((dims, pg), (dims8, pg8))):
        call = lambda k=rows, v=rows, seqs=i32(5), at=i32(5), d=d, p=p: f(d, p, k, v, seqs, at)
        for o in ({}, dict(seqs=None), dict(k=z(2, 5, 128).transpose(0, 1)), dict(v=z(5, 6, 128)[:, 2:4])):
            with pytest.raises(torch.Queued):
                call(**o)
        for o in (dict(k=z(4, 2, 128)), dict(v=z(5, 2, 64)), dict(k=z(5, 2, 256)[..., ::2]), dict(k=z(5, 2, 128, dt=torch.float32)), dict(seqs=i32(4)),
                  dict(at=i32(6)), dict(at=i32(10)[::2]), dict(at=torch.zeros(5, dtype=torch.int64)), dict(p=pg8 if p is pg else pg),
                  dict(d=B.dims(2, 1, 4, 128, 0, "bf16")), dict(d=B.dims(2, 2, 8, 64, 0, "bf16"))):
            with pytest.raises(ValueError):
                call(**o)
    for o in (z(1, 2, 128).expand(5, 2, 128), z(5, 1, 128).expand(5, 2, 128)):
        with pytest.raises(ValueError):
            B.page_read(dims, pg, o, rows, None, i32(5))
        with pytest.raises(torch.Queued):
            B.page_write(dims, pg, o, rows, None, i32(5))
    q, ws = z(3, 8, 128), z(1 << 16, dt=torch.float32)
    call = lambda p=pg, lens=i32(3), q=q, out=q, ws=ws, **o: B.paged_attn(dims, p, lens, 32, q, out, 0.1, ws, **o)
    for o in ({}, dict(more=z(3 * 8 * 2 * 132, dt=torch.float32), n_more=2)):
        with pytest.raises(torch.Queued):
            call(**o)
    for o in (dict(p=pg8), dict(lens=i32(2)), dict(lens=torch.zeros(3, dtype=torch.int64)), dict(q=z(2, 8, 128)), dict(out=z(3, 8, 128, dt=torch.float32)),
              dict(ws=ws[::2]), dict(more=z(3 * 8 * 2 * 132 - 1, dt=torch.float32), n_more=2), dict(more=z(3 * 8 * 2 * 132), n_more=2)):
        with pytest.raises(ValueError):
            call(**o)
