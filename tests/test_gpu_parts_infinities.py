"""An infinite residual coefficient of a block of four makes a rebuilt key infinite, not a NaN: a query whose
product with it is -inf gives the token no weight, one whose product is +inf has no softmax."""
import math

import numpy as np
import pytest

from gpu_cases import _pad, coef_plane_bytes
from serving_cases import attend, make_cache, unit_rows
from test_gpu_parts import _dims, log, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu

T, TOKEN, D = 200, 130, 128


def _value_at(cache, dims):
    """Byte, in the cache, of a bf16 residual coefficient of K of TOKEN in the unit of head 0."""
    at = int(cache.offsets_host[0, 0, 0]) + 2 * coef_plane_bytes(T, D, 2)
    raw = cache.buf.cpu().numpy()
    if dims.residual:
        words = raw[at:at + (T + 31) // 32 * 4].copy().view("<u4")
        t = np.arange(T)
        kept = np.flatnonzero((words[t // 32] >> (t % 32).astype(np.uint32)) & 1)
        row = int(np.flatnonzero(kept == TOKEN)[0])
        return at + _pad((T + 31) // 32 * 4) + _pad(((T + 127) // 128 + 1) * 4) + (row * 3 * D + 37) * 2
    return at + _pad(T * dims.topk * 2) + (TOKEN * dims.topk + 3) * 2


@pytest.mark.parametrize("kind,rows", [("own", 4), ("shared", 4), ("shared", 40), ("shared", 80)])
@pytest.mark.parametrize("k,ppm", [(16, None), (24, None), (0, 1000000)])
def test_an_infinite_coefficient(torch_dev, k, ppm, kind, rows):
    torch = torch_dev
    from paper_2607_06519_amd import binding as B
    G, batch = 4, rows // 4
    dims = _dims("bf16", 2, G, D, k, 2, None, ppm)
    log(f"[case] infinite coefficient k{k} ppm {ppm} {kind} {rows} rows")
    cache, _ = make_cache(torch, dims, [T], np.array([[[1, 0]]], np.uint8), 980)
    at = _value_at(cache, dims)
    cache.buf[at:at + 2] = torch.tensor([0x80, 0x7F], dtype=torch.uint8, device="cuda")       # +inf
    part = B.part(B.PART_SHARED if kind == "shared" else B.PART_OWN, cache.seq_lens, T, cache.modes, cache.offsets, cache.buf)
    ws = torch.empty(B.decode_parts_workspace(dims, batch, [part], -1) // 4 + 8, device="cuda")
    raw = cache.buf.cpu().numpy()
    for layer in range(4):
        K, V, RK, RV = unit_rows(cache, raw, 0, layer, 0, "bf16")
        channel = np.flatnonzero(np.isinf(K[TOKEN]))
        assert len(channel) == 1 and np.isfinite(np.delete(K, TOKEN, 0)).all()
        sign = np.sign(K[TOKEN, channel[0]])
        q = 2 * torch.randn(batch, 2 * G, D, generator=torch.Generator().manual_seed(layer))
        q[:, :, channel[0]] = -float(sign) * q[:, :, channel[0]].abs().clamp(min=0.1)
        q[0, 1, channel[0]] *= -1
        q = q.bfloat16().cuda()
        out = torch.zeros_like(q)
        B.decode_parts(dims, batch, [part], None, layer, q, out, 1.0 / math.sqrt(D), ws)
        got = out.double().cpu().numpy()
        want, tol = attend(q[:, :G].double().cpu().numpy().reshape(batch * G, D), [tuple(np.delete(x, TOKEN, 0) for x in (K, V, RK, RV))],
                           1.0 / math.sqrt(D), False, True)
        lost = np.zeros((batch, G), bool)
        lost[0, 1] = True
        assert np.isnan(got[:, :G][lost]).all() and np.isfinite(got[:, :G][~lost]).all() and np.isfinite(got[:, G:]).all()
        apart = np.abs(got[:, :G] - want.reshape(batch, G, D))
        assert (apart <= tol.reshape(batch, G, D))[~lost].all(), layer
