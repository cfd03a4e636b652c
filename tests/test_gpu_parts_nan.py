"""What is not a number in a query, a key or a value that a step reads comes out as such, in the rows that
read it and in no other: it is not the zero of a sequence without tokens."""
import math

import numpy as np
import pytest

from test_gpu_parts import Case, _dims, log, torch_dev  # noqa: F401

pytestmark = pytest.mark.gpu


def _check(c, layer, lost):
    """``lost [batch][Hq]``: rows that have no number; the others keep their bound."""
    got = c.run(layer).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        out, tol = c.want(layer)
    assert np.isnan(got[lost]).all(), np.argwhere(~np.isnan(got[lost]))[:4].tolist()
    assert (np.abs(got - out)[~lost] <= tol[~lost]).all()


@pytest.mark.parametrize("batch", [3, 9, 20])
@pytest.mark.parametrize("dtype", ["bf16", "f32", "bf16_e4m3"])
def test_not_a_number(torch_dev, dtype, batch):
    torch = torch_dev
    kv, G = 2, 4
    log(f"[case] NaN {dtype} batch {batch}")
    make = lambda: Case(torch, _dims(dtype, kv, G, 128, 16), dtype, batch, 970, shared=(300,), own=([(91 * s) % 130 for s in range(batch)],),
                        tail=(6, [1 + s % 6 for s in range(batch)]))
    for where in ("query", "key", "infinite logit", "value"):
        c = make()
        lost = np.zeros((batch, kv * G), bool)
        if where == "query":
            c.q[1, 5, 77] = math.nan
            lost[1, 5] = True
        elif where == "key":
            c.tail[0][2, 1, 0, 9] = math.nan
            lost[2, G:] = True
        elif where == "infinite logit":                          # exp(inf - inf)
            c.q[0, 2, 9] = 1
            c.q[0, 0, 9] = c.q[0, 1, 9] = c.q[0, 3, 9] = -1      # for these the token has no weight
            c.tail[0][0, 0, 0, 9] = math.inf
            lost[0, 2] = True
        else:
            c.tail[1][2, 0, 0] = math.nan
            lost[2, :G] = True
        if where != "infinite logit":
            _check(c, 1, lost)
            continue
        got = c.run(1).double().cpu().numpy()
        assert np.isnan(got[lost]).all()
        c.tail[0][0, 0, 0] = 0                                   # (the heads of the other group, and other sequences)
        out, tol = c.want(1)
        assert (np.abs(got - out)[1:] <= tol[1:]).all() and (np.abs(got - out)[0, G:] <= tol[0, G:]).all()
        c.tail_lens[0] = 0                                       # heads for which the infinite key weighs nothing
        out, tol = c.want(1)
        assert (np.abs(got - out)[0, [0, 1, 3]] <= tol[0, [0, 1, 3]]).all()


def test_no_token_is_still_zero(torch_dev):
    c = Case(torch_dev, _dims("bf16", 2, 4, 128, 16), "bf16", 3, 971, own=([0, 5, 0],), tail=(4, [0, 0, 2]))
    out = c.run(1)
    assert (out[0] == 0).all() and out.isfinite().all()
