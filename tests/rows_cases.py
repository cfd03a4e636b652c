"""Helpers of the tests of exact rows before their compression: attention in 64 bits with the bound that a kernel's
output keeps, pages in host memory, and what FP8 rows hold.

The bound, per output channel c of a query row (u = half an epsilon of the element type: 2^-8 in bf16, 2^-24 in fp32;
v = 2^-24; A_c = sum_t p_t |V_tc| of the exact probabilities p over the n rows that the query sees):
  * the output's own rounding: u |o_c|;
  * each probability rounded to the element type for its product: u A_c;
  * a logit is a sum of d products in fp32, off by at most (2 d + 4) v scale max_t sum_c |q_c K_tc|; products with the
    scale and the base-2 exponential add 4 v of a logit and 2^-21.  A logit off by e moves every probability by a factor
    within exp(+-2 e);
  * a sum over n rows, in tiles, waves and records, adds at most (n + 64) v of A_c."""
import numpy as np


def attend(q, K, V, scale, f32, seen=None):
    """``(out, bound)`` [n][d] of query rows q [n][d] over K and V [m][d]; ``seen [n]``: the keys of each row, the first ones."""
    n, d = q.shape
    out, bound = np.zeros((n, d)), np.zeros((n, d))
    seen = np.full(n, len(K)) if seen is None else np.asarray(seen)
    rows = np.flatnonzero(seen > 0)
    if len(rows) == 0:
        return out, bound
    q, seen, m = q[rows], seen[rows], int(seen.max())
    K, V = K[:m], V[:m]
    hidden = np.arange(m) >= seen[:, None]
    z = np.where(hidden, -np.inf, q @ K.T * scale)
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    o, A = p @ V, p @ np.abs(V)
    u, v = (2.0 ** -24, 2.0 ** -24) if f32 else (2.0 ** -8, 2.0 ** -24)
    most = np.where(hidden, 0, np.abs(q) @ np.abs(K).T).max(1)
    e = (2 * d + 4) * v * abs(scale) * most + 4 * v * np.where(hidden, 0, np.abs(z)).max(1) + 2.0 ** -21
    out[rows] = o
    bound[rows] = 1.01 * (u * np.abs(o) + (u + (seen[:, None] + 64) * v) * 1.01 * A + np.expm1(2 * e)[:, None] * 2 * A)
    return out, bound


def check(got, want, bound, what):
    bad = np.abs(got - want) > bound
    assert np.isfinite(got).all() and not bad.any(), (what, float((np.abs(got - want) - bound).max()), np.argwhere(bad)[:4].tolist())


def e4m3(code):
    """Values of E4M3 codes (uint8): sign, four bits of exponent, three of fraction."""
    code = code.astype(np.int64)
    x, f = (code >> 3) & 15, code & 7
    size = np.where(x == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (x - 10.0))
    size = np.where((code & 127) == 127, np.nan, size)
    return np.where(code >= 128, -size, size)


def held(x):
    """``(codes, exponents)`` of rows [..][d] in FP8, by search over the codes: nearest, ties to the even one."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1)
    e = np.full(top.shape, -126)
    for k in range(-126, 128):
        e = np.where(top > 448 * 2.0 ** k, k + 1, e)
    y = x / 2.0 ** e[..., None].astype(np.float64)
    grid = e4m3(np.arange(127, dtype=np.uint8))
    i = np.searchsorted(grid, np.abs(y)).clip(1, 126)
    lo, hi = grid[i - 1], grid[i]
    up = (np.abs(y) - lo > hi - np.abs(y)) | ((np.abs(y) - lo == hi - np.abs(y)) & (i % 2 == 0))
    code = np.where(up, i, i - 1) + np.where(np.signbit(y), 128, 0)
    return code.astype(np.uint8), (e + 127).astype(np.uint8)


def random_rows(torch, g, dtype, *shape):
    """Rows [..][d] of unlike sizes with a few large channels."""
    x = torch.randn(*shape, generator=g)
    x[..., :2] *= 6
    x *= 0.5 + torch.rand(*shape[:-1], 1, generator=g)
    return x.to(torch.float32 if dtype == "f32" else torch.bfloat16)


class Pool:
    """A layer's pages on the device, filled with 0xFF bytes (NaN rows), and a table of scattered pages."""

    def __init__(self, torch, dims, dtype, page, rows, spare=2, seed=0):
        from paper_2607_06519_amd import binding as B
        g = torch.Generator().manual_seed(seed)
        need = [-(-r // page) for r in rows]
        self.n_pages = sum(need) + spare
        shape = (self.n_pages, dims.n_kv_heads, page, dims.head_dim)
        dt = {"f32": torch.float32, "bf16": torch.bfloat16, "bf16_e4m3": torch.uint8}[dtype]
        self.k, self.v = (torch.full((self.n_pages * dims.n_kv_heads * page * dims.head_dim * dt.itemsize,), 255, dtype=torch.uint8,
                                     device="cuda").view(dt).view(shape) for _ in range(2))
        self.k_exp, self.v_exp = (torch.full(shape[:3], 255, dtype=torch.uint8, device="cuda") if dtype == "bf16_e4m3" else None
                                  for _ in range(2))
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(rows), max(max(need), 1)), -1, dtype=torch.int32)
        at = 0
        for s, m in enumerate(need):
            self.table[s, :m] = order[at:at + m]
            at += m
        self.table_d = self.table.cuda()
        self.dtype, self.page, self.dims = dtype, page, dims
        self.desc = B.pages(dims, self.k, self.v, self.table_d, self.k_exp, self.v_exp)

    def rows(self, which, s, n):
        """Rows 0 .. n - 1 of sequence s as the pool holds them, float64 [Hkv][n][d]."""
        t, e = getattr(self, which), getattr(self, which + "_exp")
        r = np.arange(n)
        page, slot = self.table[s].numpy()[r // self.page], r % self.page
        if e is None:
            x = t.double().cpu().numpy()[page, :, slot]
        else:
            x = e4m3(t.cpu().numpy())[page, :, slot] * 2.0 ** (e.cpu().numpy()[page, :, slot].astype(np.float64) - 127)[..., None]
        return x.transpose(1, 0, 2)
