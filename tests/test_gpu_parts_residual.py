"""The residual of V in decode over parts.  One token has the probability 1 in every row, so the output is its
rebuilt value M + R rounded once, and where the two nearly cancel a rounding of R before the sum shows.

Bound, with u = 2^-8 and v = 2^-24: u |o| for the output; the residual of a block of four goes in as a bf16 value
and its bf16 rest, off by u^2 |R|; the weighted sum of up to three coefficients in fp32, and the sums of the
products, by 8 v (|M| + sum_j |w_j z_j|), of which |R| holds at least a fraction: 64 v (|M| + max |R|)."""
import numpy as np
import pytest

from serving_cases import unit_rows
from test_gpu_parts import _dims, log, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu


def _layers(torch, dims, seed):
    """K and V [Hkv][1][d] of every layer; V of one layer of each block is near zero and the others alike."""
    g = torch.Generator().manual_seed(seed)
    k = [torch.randn(dims.n_kv_heads, 1, dims.head_dim, generator=g).bfloat16().cuda() for _ in range(dims.n_layers)]
    base = 1 + torch.rand(dims.n_kv_heads, 1, dims.head_dim, generator=g)
    v = [((1e-3 if i == 2 else 1.0) * (base + 0.2 * torch.randn(base.shape, generator=g))).bfloat16().cuda() for i in range(dims.n_layers)]
    return k, v


@pytest.mark.parametrize("kind,rows", [("own", 4), ("blocks", 4), ("shared", 4), ("shared", 40), ("shared", 80)])
@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3"])
@pytest.mark.parametrize("d,k,ppm", [(64, 64, None), (128, 16, None), (128, 128, None), (128, 0, 1000000)])
def test_values_of_a_block_of_four(torch_dev, d, k, ppm, dtype, kind, rows):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    from paper_2607_06519_amd.cache import CompressedCache
    kv, G = 2, 4
    batch = rows // G
    dims = _dims(dtype, kv, G, d, k, 2, None, ppm)
    log(f"[case] V's residual {dtype} d{d} k{k} {kind} {rows} rows")
    cache = CompressedCache(dims, [1], np.ones((1, 1, kv), np.uint8))
    scores = torch.ones(1, kv, 1, device="cuda") if ppm else None
    cache.compress(0, *_layers(torch, dims, d + k), token_scores=scores)
    one = dict(blocks=torch.zeros(1, kv, 1, dtype=torch.int32, device="cuda"), counts=torch.ones(1, kv, dtype=torch.int32, device="cuda"), n_sel=1)
    part = B.part({"own": B.PART_OWN, "blocks": B.PART_BLOCKS, "shared": B.PART_SHARED}[kind], cache.seq_lens, 1, cache.modes, cache.offsets,
                  cache.buf, **(one if kind == "blocks" else {}))
    ws = torch.empty(B.decode_parts_workspace(dims, batch, [part], -1) // 4 + 8, device="cuda")
    q = torch.randn(batch, kv * G, d, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    raw = cache.buf.cpu().numpy()
    smallest = 1.0
    for layer in range(4):
        out = torch.zeros_like(q)
        B.decode_parts(dims, batch, [part], None, layer, q, out, 0.1, ws)
        got = out.double().cpu().numpy().reshape(batch, kv, G, d)
        for h in range(kv):
            _, V, _, R = (x[0] if len(x) else x for x in unit_rows(cache, raw, 0, layer, h, dtype))
            tol = 2.0 ** -8 * np.abs(V) + 2.0 ** -16 * np.abs(R) + 64 * 2.0 ** -24 * (np.abs(V - R) + np.abs(R).max())
            assert (np.abs(got[:, h] - V) <= tol).all(), (layer, h, float((np.abs(got[:, h] - V) - tol).max()))
            if layer == 2:
                smallest = min(smallest, float((tol / np.maximum(np.abs(R), 1e-9))[np.abs(R) > 0.1].min()))
    # (not a bound of the kernel's: R rounded once is off by up to 2^-8 |R|, which the case has to be able to tell)
    assert smallest < 2.0 ** -9


@pytest.mark.parametrize("kind,rows", [("own", 4), ("blocks", 4), ("shared", 4), ("shared", 40), ("shared", 80)])
@pytest.mark.parametrize("dtype", ["bf16", "bf16_e4m3"])
@pytest.mark.parametrize("d,k,ppm", [(64, 8, None), (128, 16, None), (128, 24, None), (128, 128, None), (128, 0, 300000), (64, 0, 1000000)])
def test_one_token_among_many(torch_dev, d, k, ppm, dtype, kind, rows):
    """Every query is a multiple of one token's key, so far ahead of the others that their probabilities are zero: the
    output is that token's value, wherever in the tiles it lies.  (The sum of probabilities is off by the rounding of
    its logit z: v |z|, twice over.)"""
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    from paper_2607_06519_amd.cache import CompressedCache
    kv, G, T = 2, 4, 219
    batch = rows // G
    dims = _dims(dtype, kv, G, d, k, 2, None, ppm)
    log(f"[case] one token of {T}, {dtype} d{d} k{k} ppm {ppm} {kind} {rows} rows")
    g = torch.Generator().manual_seed(d + k)
    base = 1 + torch.rand(kv, T, d, generator=g)
    keys = [torch.randn(kv, T, d, generator=g).bfloat16().cuda()] * 4
    vals = [((1e-3 if i == 2 else 1.0) * (base + 0.2 * torch.randn(base.shape, generator=g))).bfloat16().cuda() for i in range(4)]
    cache = CompressedCache(dims, [T], np.ones((1, 1, kv), np.uint8))
    cache.compress(0, keys, vals, token_scores=torch.rand(1, kv, T, generator=g).cuda() if ppm else None)
    nb = -(-T // 64)
    lists = dict(blocks=torch.arange(nb, dtype=torch.int32, device="cuda").flip(0).expand(1, kv, nb).contiguous(),
                 counts=torch.full((1, kv), nb, dtype=torch.int32, device="cuda"), n_sel=nb)
    part = B.part({"own": B.PART_OWN, "blocks": B.PART_BLOCKS, "shared": B.PART_SHARED}[kind], cache.seq_lens, T, cache.modes, cache.offsets,
                  cache.buf, **(lists if kind == "blocks" else {}))
    ws = torch.empty(B.decode_parts_workspace(dims, batch, [part], -1) // 4 + 8, device="cuda")
    raw = cache.buf.cpu().numpy()
    for layer in (0, 2):
        units = [unit_rows(cache, raw, 0, layer, h, dtype) for h in range(kv)]
        for first in range(0, T, rows if kind == "shared" else 37):
            at = (first + 53 * np.arange(rows)) % T                # the rows' tokens, all over the tiles
            if kind == "shared" and first > 3 * rows:
                break
            q = torch.from_numpy(np.stack([12 * u[0][at] for u in units]).astype(np.float32)).bfloat16()      # [kv][rows][d]
            z = np.stack([q[h].double().numpy() @ units[h][0].T for h in range(kv)])
            ahead = z[:, np.arange(rows), at]
            z[:, np.arange(rows), at] = -np.inf
            assert (ahead - z.max(2) > 110).all()                  # exp(-110) is zero beside 1 in fp32
            q = q.view(kv, batch, G, d).transpose(0, 1).reshape(batch, kv * G, d).cuda()
            out = torch.zeros_like(q)
            B.decode_parts(dims, batch, [part], None, layer, q, out, 1.0, ws)
            got = out.double().cpu().numpy().reshape(batch, kv, G, d).transpose(1, 0, 2, 3).reshape(kv, rows, d)
            for h in range(kv):
                V, R = units[h][1][at], units[h][3][at]
                tol = 2.0 ** -8 * np.abs(V) + 2.0 ** -16 * np.abs(R) + 64 * 2.0 ** -24 * (np.abs(V - R) + np.abs(R).max(1, keepdims=True))
                tol = tol + 2 * 2.0 ** -24 * np.abs(ahead[h])[:, None] * np.abs(V)
                over = np.abs(got[h] - V) - tol
                assert (over <= 0).all(), (layer, h, at[np.argwhere(over > 0)[:4, 0]].tolist(), float(over.max()))
