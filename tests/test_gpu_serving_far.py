"""Offsets past 32 bits in every operator of a serving step: rows, segments and tails that lie
gigabytes behind their tensors' first bytes."""
import numpy as np
import pytest

from serving_cases import attend, make_cache, unit_rows
from test_gpu_parts import _dims, _modes, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu

GB = 1 << 30


def test_rope_append_into_a_long_cache(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    kv, d, cap, n = 8, 128, 2_300_000, 3                           # 4.7 GB a tensor
    print("[case] rows past 4 GB", flush=True)
    dims = B.dims(2, kv, kv, d, 0, "bf16")
    k, v = (torch.zeros(1, kv, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = torch.randn(n, 3 * kv, d, device="cuda").bfloat16()
    rows = torch.tensor([cap - 1, 5, cap // 2], dtype=torch.int32, device="cuda")
    seqs = torch.zeros(n, dtype=torch.int32, device="cuda")
    rope = B.rope(0, torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"))
    q = torch.empty(n, kv, d, dtype=torch.bfloat16, device="cuda")
    B.rope_append(dims, rope, *x.split(kv, 1), q, seqs, rows, k, v)
    for t, at in ((k, kv), (v, 2 * kv)):
        assert torch.equal(t[0, :, rows.long()], x[:, at:at + kv].transpose(0, 1))
        t[0, :, rows.long()] = 0
        assert not t.any()


def test_bounds_of_long_keys(torch_dev):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    kv, d, T = 2, 128, 9_000_000                                   # 4.6 GB a layer
    print("[case] keys past 4 GB", flush=True)
    dims = B.dims(2, kv, kv, d, 0, "bf16")
    k = torch.zeros(kv, T, d, dtype=torch.bfloat16, device="cuda")
    k[1, T - 1], k[1, T - 65, 3], k[0, 70, 5] = 2.0, -3.0, 4.0
    nb = -(-T // 64)
    out = torch.full((2, kv, nb, 2, d), 9.0, dtype=torch.bfloat16, device="cuda")
    B.key_bounds(dims, T, [k, k], list(out), nb)
    for l in range(2):
        assert (out[l, 1, nb - 1, 1] == 2).all() and (T % 64 == 1 or not out[l, 1, nb - 1, 0].any())
        assert out[l, 1, (T - 65) // 64, 0, 3] == -3 and out[l, 0, 1, 1, 5] == 4
    assert int((out != 0).sum()) == 2 * (d * (2 if T % 64 == 1 else 1) + 2)


def test_parts_far_behind_their_buffers(torch_dev):
    """Segments 5 GB behind the cache's first byte, and the last head of a tail 7 GB behind its first."""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    for dtype, sched in (("bf16", 0), ("bf16_e4m3", 2)):
        print(f"[case] far segments {dtype}", flush=True)
        dims = _dims(dtype, 8, 2, 128, 16, sched)
        own = make_cache(torch, dims, [300, 77], _modes(dims, 2, 1), 950)[0]
        shared = make_cache(torch, dims, [500], _modes(dims, 1, 2), 951)[0]
        buf = torch.zeros(5 * GB + own.buf.numel() + shared.buf.numel() + 512, dtype=torch.uint8, device="cuda")
        at = 5 * GB
        parts = []
        for kind, c in ((B.PART_OWN, own), (B.PART_SHARED, shared)):
            n = c.buf.numel()
            buf[at:at + n] = c.buf
            c.far = c.offsets + at
            parts.append(B.part(kind, c.seq_lens, c.max_seq_len, c.modes, c.far, buf))
            at += -(-n // 256) * 256
        cap = 2_100_000                                            # 0.5 GB a head and sequence
        k, v = (torch.zeros(2, 8, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        g = torch.Generator().manual_seed(952)
        for t in (k, v):
            t[:, :, :40] = torch.randn(2, 8, 40, 128, generator=g).bfloat16().cuda()
            t[:, :, 40:100] = float("nan")
        lens = torch.tensor([40, 9], dtype=torch.int32, device="cuda")
        tail = B.Tail(lens.data_ptr(), cap, k.data_ptr(), v.data_ptr())
        q = (2 * torch.randn(2, 16, 128, generator=g)).bfloat16().cuda()
        out = torch.empty_like(q)
        ws = torch.empty(B.decode_parts_workspace(dims, 2, parts, cap) // 4 + 8, device="cuda")
        B.decode_parts(dims, 2, parts, tail, 1, q, out, 0.09, ws)
        raw = [c.buf.cpu().numpy() for c in (own, shared)]
        got, qs = out.double().cpu().numpy(), q.double().cpu().numpy()
        for s in range(2):
            for h in range(8):
                n = int(lens[s])
                tk, tv = (t[s, h, :n].double().cpu().numpy() for t in (k, v))
                have = [unit_rows(own, raw[0], s, 1, h, dtype), unit_rows(shared, raw[1], 0, 1, h, dtype), (tk, tv, 0 * tk, 0 * tv)]
                want, tol = attend(qs[s, 2 * h:2 * h + 2], have, 0.09, False, True)
                assert (np.abs(got[s, 2 * h:2 * h + 2] - want) <= tol).all(), (dtype, s, h)
        del buf, k, v
