"""PagedCache on the host: which calls it refuses and what they leave.  The library's device calls are replaced by stubs;
everything else is the class's own code on CPU tensors."""
import os

import pytest

from paper_2607_06519_amd import binding as B
from paper_2607_06519_amd import cache as C

DIMS = B.dims(2, 2, 8, 128, 0, "bf16")


@pytest.fixture
def calls(monkeypatch):
    import torch
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libfdkv.so not built")
    seen = []
    monkeypatch.setattr(C, "_torch", lambda: torch)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    for name in ("page_write", "page_read", "prompt_attn", "paged_attn", "decode_partial"):
        monkeypatch.setattr(C.B, name, lambda *a, _name=name, **k: seen.append((_name, a)))
    return seen


def _cache(batch=2, max_len=100, dims=DIMS, **o):
    return C.PagedCache(dims, batch, max_len, page=16, device="cpu", **o)


def _rows(n, heads, dtype=None):
    import torch
    return torch.zeros(n, heads, 128, dtype=dtype or torch.bfloat16)


def test_a_prompt_of_other_rows_is_refused(calls):
    """Queries, keys, values and outputs are those of the rows that have begun; a call that is refused stores nothing."""
    import torch
    c = _cache()
    rows = c.begin([5, 2])
    good = dict(q=_rows(7, 8), k=_rows(7, 2), v=_rows(7, 2))
    for bad in (dict(q=_rows(6, 8)), dict(q=_rows(8, 8)), dict(q=_rows(0, 8)), dict(q=_rows(7, 4)), dict(q=_rows(7, 8)[..., :64]), dict(k=_rows(6, 2)),
                dict(k=_rows(7, 8)), dict(v=_rows(8, 2)), dict(v=_rows(7, 1)), dict(q=_rows(7, 8).flatten(1)), dict(out=_rows(6, 8)), dict(out=_rows(8, 8))):
        with pytest.raises(ValueError):
            c.prompt(rows, 0, **{**good, **bad})
    assert not calls
    c.prompt(rows, 0, **good)
    c.prompt(rows, 1, **good, out=torch.empty_like(good["q"]))
    assert [x[0] for x in calls] == ["page_write", "prompt_attn"] * 2
    c.end(rows)
    none = c.begin([0, 0])
    for bad in (dict(q=_rows(1, 8)), dict(k=_rows(1, 2)), dict(out=_rows(1, 8))):
        with pytest.raises(ValueError):
            c.prompt(none, 0, **{**dict(q=_rows(0, 8), k=_rows(0, 2), v=_rows(0, 2)), **bad})
    assert c.prompt(none, 0, _rows(0, 8), _rows(0, 2), _rows(0, 2)).shape == (0, 8, 128)


def test_rows_that_cannot_begin_take_no_pages(calls, monkeypatch):
    """A begin that is refused, or fails on its way, leaves the pages where they were."""
    import torch
    c = _cache(2, 1000)
    rows = c.begin([40, 3])
    c.end(rows)
    free, table = list(c.free), c.table.clone()

    def unchanged():
        assert c.free == free and [len(h) for h in c.held] == [3, 1] and torch.equal(c.table, table) and c.lens_host == [40, 3]

    def refuse(*a):
        raise B.FdkvError(-2, "fdkv_prompt_attn_workspace")
    with monkeypatch.context() as m:
        m.setattr(C.B, "prompt_attn_workspace", refuse)
        with pytest.raises(B.FdkvError):
            c.begin([500, 0])
    unchanged()
    make, made = torch.tensor, []

    def second(*a, **k):                                     # the second sequence's pages cannot be put into the table
        made.append(a)
        if len(made) == 2:
            raise MemoryError
        return make(*a, **k)
    with monkeypatch.context() as m:
        m.setattr(torch, "tensor", second)
        with pytest.raises(MemoryError):
            c.begin([30, 30])
    unchanged()
    c.end(c.begin([500, 60]))
    assert sorted(c.free + c.held[0] + c.held[1]) == list(range(c.n_pages)) and c.lens_host == [540, 63]


def test_more_rows_than_a_call_takes(calls, monkeypatch):
    """A prompt's rows are stored, and earlier ones gathered, in calls of as many rows as one takes."""
    monkeypatch.setattr(C.B, "MAX_PAGE_GROUPS", 4, raising=False)   # 16 rows of two heads
    c = _cache(2, 1000)
    for counts in ([33, 0], [7, 10]):
        rows = c.begin(counts)
        n = sum(counts)
        calls.clear()
        c.prompt(rows, 1, _rows(n, 8), _rows(n, 2), _rows(n, 2))
        for name, total, heads_first in (("page_write", n, False), ("page_read", 50, True)):
            mine = [a for x, a in calls if x == name]
            if name == "page_read" and counts[0] == 33:
                assert not mine
                continue
            assert [len(a[5]) for a in mine] == [16] * (total // 16) + [total % 16]
            assert all(a[2].shape == a[3].shape == (len(a[5]), 2, 128) and len(a[4]) == len(a[5]) and a[1] is c.pools[1] for a in mine)
            if heads_first:
                assert [int(r) for a in mine for r in a[5]] == [*range(40), *range(10)]
                base = mine[0][2].data_ptr()
                assert [a[2].data_ptr() - base for a in mine] == [2 * 128 * 16 * i for i in range(len(mine))]
        c.end(rows)
    calls.clear()
    k, v = c.read(0, 0)
    assert k.shape == v.shape == (2, 40, 128) and [len(a[5]) for _, a in calls] == [16, 16, 8]
    dims = B.dims(2, 8, 8, 128, 0, "bf16")                    # the limit is the library's
    import ctypes
    two = (ctypes.c_int64 * 2)(1024, 128)
    pages = B.Pages(1, 16, 1, 1, 1 << 20, 1 << 20, 1 << 20, None, None)
    monkeypatch.undo()
    most = B.MAX_PAGE_GROUPS // 8 * 8
    lib = B.load()
    for n, status in ((most + 1, -2), (most, -1)):            # (no rows' addresses: refused for that alone)
        assert lib.fdkv_page_read(ctypes.byref(dims), ctypes.byref(pages), n, None, two, None, two, None, None, None) == status


def test_cancelled_rows_and_steps(calls):
    """What has begun can be given up, and leaves the sequences, the pages and the table as they were."""
    import torch
    c = _cache(3, 100, n_pages=13)
    with pytest.raises(RuntimeError):
        c.cancel()
    c.end(c.begin([40, 16, 0]))
    free, table = list(c.free), c.table.clone()

    def unchanged():
        assert c.free == free and [len(h) for h in c.held] == [3, 1, 0] and c.lens_host == [40, 16, 0] and torch.equal(c.table, table)
        assert c._open is None and c.active == [False] * 3
    rows = c.begin([30, 20, 50])
    calls.clear()
    c.prompt(rows, 0, _rows(100, 8), _rows(100, 2), _rows(100, 2))
    c.cancel()
    unchanged()
    for late in (lambda: c.prompt(rows, 1, _rows(100, 8), _rows(100, 2), _rows(100, 2)), lambda: c.end(rows), c.cancel):
        with pytest.raises(RuntimeError):
            late()
    c.begin_step([True, True, True])
    assert c.pos.tolist() == [40, 16, 0] and len(c.held[1]) == 2
    c.append(0, _rows(3, 2), _rows(3, 2))
    c.cancel()
    unchanged()
    assert c.pos.tolist() == [-1] * 3 and c.lens.tolist() == [0] * 3
    for late in (c.advance, lambda: c.append(1, _rows(3, 2), _rows(3, 2)), lambda: c.decode(1, _rows(3, 8))):
        with pytest.raises(RuntimeError):
            late()
    c.release(0)
    c.end(c.begin([1, 80, 90]))
    assert sorted(c.free + sum(c.held, [])) == list(range(13)) and c.lens_host == [1, 96, 90]


def _prefix(lens, dims=DIMS):
    import numpy as np
    return C.CompressedCache(dims, lens, np.zeros((len(lens), len(B.blocks(dims)[0]), dims.n_kv_heads), np.uint8), device="cpu")


def test_the_first_step_behind_a_prefix(calls, monkeypatch):
    """A sequence that holds tokens of the prefix and no rows is not passed over unless the caller says so."""
    import torch
    c, prefix = _cache(3, 100), _prefix([300, 0, 20])
    q, kv = _rows(3, 8), _rows(3, 2)
    c.begin_step()                                           # (no sequence holds a row)
    with pytest.raises(RuntimeError, match="prefix"):
        c.decode(0, q, prefix=prefix)
    assert not calls
    c.decode(0, q)                                           # without it there is nothing to pass over
    c.cancel()
    c.begin_step(prefix=prefix)
    assert c.active == [True, False, True] and c.pos.tolist() == [0, -1, 0] and c.lens.tolist() == [1, 0, 1]
    c.append(0, kv, kv)
    c.decode(0, q, prefix=prefix)
    c.advance()
    c.begin_step()                                           # both hold a row now
    c.decode(0, q, prefix=prefix)
    c.advance()
    c.release(2)
    c.begin_step([True, False, False])                       # sequence 2 has ended: the caller says so
    c.decode(0, q, prefix=prefix)
    c.advance()
    c.begin_step([True, False, False], prefix=prefix)
    assert c.active == [True, False, False]
    c.decode(0, q, prefix=prefix)
    c.advance()
    with pytest.raises(ValueError):
        c.begin_step(prefix=_prefix([1, 2]))
    assert c._open is None and c.lens_host == [4, 0, 0]
    # a captured step reads its prefix at every replay
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    c.decode(0, q, prefix=prefix)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    with pytest.raises(RuntimeError, match="prefix"):
        c.begin_step()
    assert c._open is None and c.lens_host == [4, 0, 0]
    c.begin_step(prefix=prefix)
    assert c.active == [True, False, True]


def test_a_step_of_another_batch_is_refused(calls):
    """Queries and outputs of more sequences than the cache's would keep rows that nothing writes."""
    c = _cache(3, 100)
    c.begin_step([True] * 3)
    for bad in (dict(q=_rows(4, 8)), dict(q=_rows(2, 8)), dict(q=_rows(3, 4)), dict(q=_rows(3, 8), out=_rows(4, 8)), dict(q=_rows(3, 8), out=_rows(2, 8))):
        with pytest.raises(ValueError):
            c.decode(0, **bad)
    assert not calls
    assert c.decode(0, _rows(3, 8)).shape == (3, 8, 128) and [x[0] for x in calls] == ["paged_attn"]
    assert c.decode(0, _rows(3, 8).flatten(1)).shape == (3, 1024)
