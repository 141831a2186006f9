"""lsam_recurrence where states or inputs are infinite: by the definition, step by step, a state that is infinite stays so as long as the
gates are positive, however small the product of many of them is.  Values are compared where the definition's are finite
with the bounds that the finite tests derive; infinities and NaN have to be where the definition has them."""
import math

import numpy as np
import pytest
import torch

from paper_2509_03110_amd import ops
from test_gpu_recurrence import B16, DEV, F32, make, np64

pytestmark = pytest.mark.gpu


def steps(f, x, h0, dh, dlast):
    """A sequence [T, D] in 64 bits; gates of at most |f| = 80, which fp32 has as well."""
    T, D = f.shape
    with np.errstate(invalid="ignore"):
        a, b = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(f))
        h = np.zeros((T + 1, D))
        h[0] = h0
        for t in range(T):
            h[t + 1] = a[t] * h[t] + b[t] * x[t]
        dx, df, e = np.zeros((T, D)), np.zeros((T, D)), dlast.copy()
        for t in range(T - 1, -1, -1):
            d = dh[t] + e
            dx[t], df[t], e = b[t] * d, a[t] * b[t] * d * (h[t] - x[t]), a[t] * d
    return h, df, dx, e


def same(got, want, what):
    g = np64(got)
    assert np.array_equal(np.isnan(g), np.isnan(want)), what
    assert np.array_equal(np.isposinf(g), np.isposinf(want)) and np.array_equal(np.isneginf(g), np.isneginf(want)), what
    ok = np.isfinite(want)
    # the states of 128 rows at most are formed from rounded products: 2^-7 of the largest covers bfloat16's rounding and theirs
    size = np.abs(want[ok]).max(initial=1.0)
    assert np.all(np.abs(g[ok] - want[ok]) <= 2.0 ** -7 * size), what


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("S,T,D,packed", [(2, 1, 9, False), (3, 14, 5, False), (2, 100, 70, False), (130, 300, 130, False), (1, 5000, 6, False), (3, 1700, 6, True)])
def test_infinite_states_stay_infinite(dtype, S, T, D, packed):
    f, x, h0, dh, dlast = make((S, T, D), S, dtype, seed=T + D)
    f[:, :, 0], f[:, :, 1 % D], f[:, :, 2 % D] = -12.0, -80.0, 3.0      # products of 16 gates underflow; of one nearly; of some hundred
    h0[0, :4], h0[S - 1, 3:5] = math.inf, -math.inf
    dlast[S - 1, :4], dlast[0, 3:5] = -math.inf, math.inf
    x[S - 1, T // 2, 0], dh[0, T // 3, 2] = math.inf, math.inf
    x[0, T // 2, 3], dh[S - 1, T // 3, 3] = -math.inf, math.inf        # against an infinite state of the other sign: NaN
    if packed:
        off = torch.tensor([T * k for k in range(S + 1)], dtype=torch.int64, device=DEV)
        flat = [t.view(S * T, D) for t in (f, x, dh)]
        r = ops.recurrence(flat[0], flat[1], h0=h0, offsets=off, save=True)
        g = ops.recurrence_backward(flat[0], flat[1], flat[2], r.states, h0=h0, dlast=dlast, offsets=off)
    else:
        r = ops.recurrence(f, x, h0=h0, save=True)
        g = ops.recurrence_backward(f, x, dh, r.states, h0=h0, dlast=dlast)
    h, df, dx = (t.view(S, T, D) for t in (r.h, g[0], g[1]))
    for i in (0, S // 2, S - 1):
        wh, wf, wx, we = steps(np64(f[i]), np64(x[i]), np64(h0[i]), np64(dh[i]), np64(dlast[i]))
        same(h[i], wh[1:], "h")
        same(r.last[i], wh[-1], "last")
        same(df[i], wf, "df")
        same(dx[i], wx, "dx")
        same(g[2][i], we, "dh0")


@pytest.mark.parametrize("T", [3, 5000])
def test_a_gate_of_zero_takes_an_infinite_state_for_nan(T):
    f, x, h0, dh, dlast = make((1, T, 2), 1, F32, seed=T)
    h0[:] = math.inf
    f[0, T // 2, 1] = -math.inf                                      # 0 x inf
    r = ops.recurrence(f, x, h0=h0)
    assert bool((r.h[0, :, 0] == math.inf).all()) and bool((r.h[0, :T // 2, 1] == math.inf).all()) and bool(r.h[0, T // 2:, 1].isnan().all())
