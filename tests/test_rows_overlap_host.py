"""Rows that a page_read writes do not overlap (the tensors are on the CPU, and no kernel runs)."""
import os

import pytest

from paper_2607_06519_amd import binding as B


def test_rows_that_are_written_do_not_overlap(monkeypatch):
    import torch
    if not os.path.exists(B._LIB_PATH):
        pytest.skip("libfdkv.so not built")
    B.load()

    class Queued(Exception):
        pass

    def queued(*a):
        raise Queued
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", queued, raising=False)
    hkv, hd = 3, 64
    dims = B.dims(2, hkv, hkv, hd, 0, "bf16")
    zeros = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    pages = B.pages(dims, zeros(4, hkv, 16, hd), zeros(4, hkv, 16, hd), torch.zeros(1, 4, dtype=torch.int32))
    many = zeros(1 << 16)
    for n in (1, 2, 5):
        at = torch.zeros(n, dtype=torch.int32)
        for by_n in (0, 32, hd, 2 * hd, hkv * hd, n * hd, 4 * hd, 10 * hd):
            for by_m in (0, 32, hd, 2 * hd, hkv * hd, n * hd, 4 * hd, 10 * hd):
                out, other = many.as_strided((n, hkv, hd), (by_n, by_m, 1)), zeros(n, hkv, hd)
                places = sorted(i * by_n + j * by_m for i in range(n) for j in range(hkv))
                apart = all(b - a >= hd for a, b in zip(places, places[1:]))
                # (rows of one axis between those of the other are refused, too)
                nested = n == 1 or by_n >= (hkv - 1) * by_m + hd or by_m >= (n - 1) * by_n + hd
                for k, v in ((out, other), (other, out)):
                    with pytest.raises(Queued if apart and nested else ValueError):
                        B.page_read(dims, pages, k, v, None, at)
                    with pytest.raises(Queued):              # rows that are read may
                        B.page_write(dims, pages, k, v, None, at)
