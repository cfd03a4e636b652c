"""fdkv_decode_parts where many query rows share a span: the kernels of 64 and of
128 columns for every type and residual kind, the workgroups that a head gets by its
mode, lengths below their bounds, and scales of any sign.  The oracle and its bound
are those of serving_cases."""
import numpy as np
import pytest

import test_gpu_parts as parts
from test_gpu_parts import KINDS, Case, _dims, _kind, log, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [64, 128])
@pytest.mark.parametrize("name", list(KINDS))
def test_wide_kernels(torch_dev, name, rows):
    """Up to 64 rows go by 32 or 64, more than 64 by 128 (fp32: up to 112 rows by 16); ragged in their last tile."""
    dims, dtype, layers = _kind(name)
    G = dims.n_q_heads // dims.n_kv_heads
    batch = {64: 40, 128: 120}[rows] // G + 1
    log(f"[case] wide {name} {batch} x {G}")
    layer = dims.n_layers - 1
    Case(torch_dev, dims, dtype, batch, 300 + rows, shared=(219,), tail=(9, [s % 10 for s in range(batch)])).check((layer,), name)


def _one_of(mode, others):
    def modes(dims, n, seed):
        from paper_2607_06519_amd import binding as B
        m = np.full((n, len(B.blocks(dims)[0]), dims.n_kv_heads), others, np.uint8)
        m[:, :, seed % dims.n_kv_heads] = mode
        return m
    return modes


@pytest.mark.parametrize("kv", [1, 3, 8, 11, 64, 65])
@pytest.mark.parametrize("mode,others", [(1, 0), (0, 1), (2, 1), (1, 1), (0, 2)])
def test_workgroups_by_mode(torch_dev, monkeypatch, kv, mode, others):
    """One head unlike the others, all alike, and more heads than the workgroups are dealt over."""
    monkeypatch.setattr(parts, "_modes", _one_of(mode, others))
    T = 1500 if kv < 20 else 200
    log(f"[case] modes {kv} heads, one {mode} among {others}, T {T}")
    for batch, dtype, sched in ((3, "bf16", 0), (20, "bf16_e4m3", 2)):
        dims = _dims(dtype, kv, 1, 64, 8, sched)
        Case(torch_dev, dims, dtype, batch, 400 + kv, shared=(T,), tail=(5, [s % 6 for s in range(batch)])).check((1,), f"{dtype} {kv}")


@pytest.mark.parametrize("dtype", ["bf16", "f32", "bf16_e4m3"])
def test_lengths_below_their_bounds(torch_dev, dtype):
    """A launch sized for longer parts (a graph captured for the longest) reads what the lengths say."""
    torch = torch_dev
    dims = _dims(dtype, 3, 4, 128, 16)
    for batch in (2, 9, 20):
        lens = [[(37 * s) % 200 for s in range(batch)], [(53 * s) % 150 for s in range(batch)]]
        lists = [[sorted(set([0, (T - 1) // 64])) if T else [] for _ in range(3)] for T in lens[1]]
        c = Case(torch, dims, dtype, batch, 500 + batch, shared=(411,), own=(lens[0],), blocks=(lens[1], lists, 4),
                 tail=(40, [(11 * s) % 41 for s in range(batch)]))
        log(f"[case] bounds {dtype} batch {batch}")
        B = c.B
        for p, most in zip(c.parts, (20000, 3000, 5000)):
            p.max_seq_len = most
        c.ws = torch.full((B.decode_parts_workspace(dims, batch, c.parts, c.cap) // 4 + 8,), float("nan"), device="cuda")
        c.check((0, 1), dtype)


@pytest.mark.parametrize("scale", [0.0, -0.07, 1e-30, 1.5])
def test_scales(torch_dev, scale):
    for dtype, batch in (("bf16", 3), ("bf16", 30), ("f32", 9)):
        c = Case(torch_dev, _dims(dtype, 2, 4, 64, 8, 2), dtype, batch, 600, shared=(300,), own=([(91 * s) % 130 for s in range(batch)],),
                 tail=(6, [s % 7 for s in range(batch)]), qscale=1.0)
        c.scale = scale
        log(f"[case] scale {scale} {dtype} {batch}")
        c.check((1,), f"{dtype} {scale}")


def test_same_call_same_bits(torch_dev):
    """Nothing is summed in an order that time decides."""
    torch = torch_dev
    dims = _dims("bf16", 8, 4, 128, 16)
    c = Case(torch, dims, "bf16", 16, 700, shared=(5000,), own=([(311 * s) % 900 for s in range(16)],), tail=(64, [4 * s for s in range(16)]))
    first = c.run(1)
    for _ in range(3):
        c.ws.fill_(float("nan"))
        assert torch.equal(c.run(1), first)


def test_calls_on_two_streams_at_once(torch_dev):
    """A workspace each: calls that overlap do not meet."""
    torch = torch_dev
    dims = _dims("bf16", 4, 4, 128, 16)
    cases = [Case(torch, dims, "bf16", 8, 710 + i, shared=(3000,), tail=(20, [2 * s for s in range(8)])) for i in range(2)]
    want = [c.run(1) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.zeros_like(c.q) for _ in range(6)] for c in cases]
    torch.cuda.synchronize()
    for i in range(6):
        for c, s, o in zip(cases, streams, outs):
            c.run(1, o[i], stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, x) for x in o)


@pytest.mark.parametrize("kv", [2, 5, 8, 64])
@pytest.mark.parametrize("dtype,sched", [("bf16_e4m3", 2), ("bf16", 0)])
def test_heads_in_the_order_of_their_cost(torch_dev, monkeypatch, kv, dtype, sched):
    """More workgroups than CUs, walks of 16 tiles and more: every head is taken once, whatever the modes are."""
    def modes(dims, n, seed):
        from paper_2607_06519_amd import binding as B
        rng = np.random.default_rng(seed)
        m = rng.integers(0, 3, (n, len(B.blocks(dims)[0]), dims.n_kv_heads)).astype(np.uint8)
        m[0], m[-1] = 1, 2                                        # all alike
        return m
    monkeypatch.setattr(parts, "_modes", modes)
    batch = -(-300 // kv)
    log(f"[case] order {dtype} {kv} heads, {batch} sequences")
    lens = [300 + (97 * s) % 300 for s in range(batch)]
    dims = _dims(dtype, kv, 1, 64, 8, sched)
    Case(torch_dev, dims, dtype, batch, 800 + kv, own=(lens,)).check((1,), f"{dtype} {kv}")
