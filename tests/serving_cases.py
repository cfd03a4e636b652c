"""Helpers of the tests of decode over parts: caches of random inputs, their rows
read back and rebuilt in 64 bits, and attention with the bound that a kernel's
output keeps.

The bound, per output channel c of a query row (u = half an epsilon of the
element type: 2^-8 in bf16, 2^-24 in fp32; v = 2^-24; A_c = sum_t p_t |V_tc| of
the exact probabilities p):
  * the output's own rounding: u |o_c|;
  * each probability rounded to the element type for its product: u A_c;
  * of a block of four in bf16, V's residual rounded to bf16 once: u sum_t p_t |R_tc|,
    and K's to a bf16 pair: a logit off by u^2 scale max_t sum_c |q_c R_tc|;
  * fp32: a logit is a sum of d products (and as many of the residual), off by
    at most (2 d + 4) v scale max_t sum_c |q_c| (|K_tc| + |R_tc|); products with
    the scale and the base-2 exponential add 4 v of a logit and 2^-21;
    a sum over n tokens, in tiles, waves and records, adds at most (n + 64) v of A_c.
  A logit off by e moves every probability by a factor within exp(+-2 e).
"""
import math

import numpy as np

import oracle as O

from gpu_cases import BYTES, TYPES, _pad, coef_plane_bytes, shared_plane, unpack_unit, values


def random_layers(torch, dims, T, seed, B=None):
    """K and V of every layer, lists of [Hkv][T][d] device tensors; neighbouring layers alike, as in a model."""
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dims.dtype == 0 else torch.bfloat16
    base = torch.randn(2, dims.n_kv_heads, T, dims.head_dim, generator=g)
    out = ([], [])
    for _ in range(dims.n_layers):
        for i in range(2):
            x = 0.8 * base[i] + 0.6 * torch.randn(base[i].shape, generator=g)
            out[i].append(x.to(dt).cuda())
    return out


def make_cache(torch, dims, lens, modes, seed):
    """A CompressedCache of random inputs in a buffer that held 0xFF (NaN) bytes before."""
    from paper_2607_06519_amd import binding as B
    from paper_2607_06519_amd.cache import CompressedCache
    cache = CompressedCache(dims, lens, modes)
    cache.buf.fill_(0xFF)
    keys = []
    for s, T in enumerate(lens):
        if T == 0:
            keys.append(None)
            continue
        k, v = random_layers(torch, dims, T, seed + 17 * s)
        scores = None
        if dims.residual == B.RES_TOKENS:
            g = torch.Generator().manual_seed(seed + 5 + s)
            scores = torch.rand(len(cache.block_size), dims.n_kv_heads, T, generator=g).cuda()
        cache.compress(s, k, v, token_scores=scores)
        keys.append(k)
    torch.cuda.synchronize()
    return cache, keys


def _tokens_unit(raw, off, T, d, dtype, B, ppm):
    ti, tc = TYPES[dtype]
    c = BYTES[tc]
    coef = coef_plane_bytes(T, d, c)
    n = -(-T * ppm // 1000000)
    u = {"MK": shared_plane(raw, off, T, d, dtype), "MV": shared_plane(raw, off + coef, T, d, dtype)}
    o = off + 2 * coef
    words = raw[o:o + (T + 31) // 32 * 4].copy().view("<u4")
    t = np.arange(T)
    u["TS"] = np.flatnonzero((words[t // 32] >> (t % 32).astype(np.uint32)) & 1)
    assert len(u["TS"]) == n
    o += _pad((T + 31) // 32 * 4) + _pad(((T + 127) // 128 + 1) * 4)
    for which in "KV":
        m = n * (B - 1) * d * c
        u["H" + which] = values(raw[o:o + m].copy(), tc).reshape(n, B - 1, d)
        o += _pad(m)
    return u


def unit_rows(cache, raw, s, layer, head, dtype):
    """(K~, V~, R_K, R_V) [T][d] in float64 of a unit at a layer, from the cache's bytes; R: what the residual adds."""
    dm = cache.dims
    b = next(i for i, (f, n) in enumerate(zip(cache.block_first, cache.block_size)) if f <= layer < f + n)
    B, pos = int(cache.block_size[b]), layer - int(cache.block_first[b])
    T, d, off = cache.seq_lens_host[s], dm.head_dim, int(cache.offsets_host[s, b, head])
    byte = int(cache.modes_host[s, b, head])
    mode = byte & 3
    if T == 0:
        return (np.zeros((0, d)),) * 4
    if mode == O.RESIDUAL and dm.residual:
        ppm = dm.rates_ppm[byte >> 2] if dm.n_rates else dm.res_ppm
        unit = _tokens_unit(raw, off, T, d, dtype, B, ppm)
        full = [O.reconstruct_layer_tokens(unit, mode, pos, d, w, B) for w in "KV"]
    else:
        unit = unpack_unit(raw, off, mode, T, d, dm.topk, dtype, B)
        full = [O.reconstruct_layer(unit, mode, pos, d, w, B) for w in "KV"]
    if mode != O.RESIDUAL:
        return full[0], full[1], np.zeros_like(full[0]), np.zeros_like(full[1])
    return full[0], full[1], full[0] - unit["MK"], full[1] - unit["MV"]


def attend(q, parts, scale, f32, quads):
    """``(out, bound)`` [G][d] of queries q [G][d] over parts, lists of (K, V, R_K, R_V)."""
    K, V, RK, RV = (np.concatenate([p[i] for p in parts]) for i in range(4))
    n, d = K.shape
    if n == 0:
        return np.zeros(q.shape), np.zeros(q.shape)
    z = q @ K.T * scale
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    out = p @ V
    u, v = (2.0 ** -24, 2.0 ** -24) if f32 else (2.0 ** -8, 2.0 ** -24)
    A, AR = p @ np.abs(V), p @ np.abs(RV)
    aq = np.abs(q)
    M = np.abs(K) + 2 * np.abs(RK)
    e = (2 * d + 4) * v * abs(scale) * (aq @ M.T).max(1) + 4 * v * np.abs(z).max(1) + 2.0 ** -21
    if quads and not f32:
        e = e + u * u * abs(scale) * (aq @ np.abs(RK).T).max(1)
    grow = np.expm1(2 * e)[:, None]
    bound = u * np.abs(out) + (u + (n + 64) * v) * 1.01 * A + grow * 2 * A
    if quads and not f32:
        bound = bound + u * AR
    return out, bound * 1.01
