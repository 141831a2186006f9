"""lsam_adapter and its gradients against the definition in 64 bits.

Where the tolerances come from (u = 2^-24): every product of operands that are multiplied as stored (bfloat16), or in pieces of
which the six largest products are formed (fp32: what is left out is below 4 u of the product), is summed in fp32.  Sums
of n terms are off by at most n u of the sum of their absolute values in any order; the matrix units add groups of terms with
at most one rounding each, and splitting a sum only shortens it, so (n + 8) u of the sum of absolute values bounds all of them.
u = x A^T and du carry such an error into the results that they are part of.  For a result that is stored as bfloat16, u, du and the
adapters are multiplied in two pieces, 2^-16 of the low-rank term's absolute sum at most, and the result is rounded by 2^-8 of
itself."""
import math

import numpy as np
import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, B16 = torch.float32, torch.bfloat16


def n64(t):
    return t.double().cpu().numpy()


def within(got, want, bound, dtype, what):
    g = n64(got)
    tol = bound + ((2.0 ** -8 * (np.abs(want) + bound)) if dtype == B16 else U * np.abs(want)) + 1e-36
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(g - want) / tol)), np.argwhere(bad)[:4].tolist())


def reference(x, W, A, B, begin, which, scale, bias, dy):
    X, Wn, An, Bn, DY = n64(x), n64(W), n64(A), n64(B), n64(dy)
    rows, inp = X.shape
    out, rank, m = Wn.shape[0], An.shape[1], An.shape[0]
    ax, aw, ady = np.abs(X), np.abs(Wn), np.abs(DY)
    two = 2.0 ** -16 if x.dtype == B16 else 0.0
    Y, bY = X @ Wn.T, (inp + 8) * U * (ax @ aw.T)
    if bias is not None:
        Y, bY = Y + n64(bias), bY + 2 * U * np.abs(n64(bias))
    DX, bDX = DY @ Wn, (out + 8) * U * (ady @ aw)
    u, bu = np.zeros((rows, rank)), np.zeros((rows, rank))
    dA, dB = np.zeros((m, rank, inp)), np.zeros((m, out, rank))
    bA, bB = np.zeros_like(dA), np.zeros_like(dB)
    for s, a in enumerate(which):
        lo, hi = (min(max(v, 0), rows) for v in (begin[s], begin[s + 1]))
        if not 0 <= a < m or lo >= hi:
            continue
        r = slice(lo, hi)
        aA, aB = np.abs(An[a]), np.abs(Bn[a])
        su = ax[r] @ aA.T
        u[r], bu[r] = X[r] @ An[a].T, (inp + 8) * U * su
        Y[r] += scale * (u[r] @ Bn[a].T)
        bY[r] += abs(scale) * ((bu[r] + ((rank + 12) * U + two) * su) @ aB.T)
        sdu = abs(scale) * (ady[r] @ aB)
        du, bdu = scale * (DY[r] @ Bn[a]), (out + 10) * U * sdu
        DX[r] += du @ An[a]
        bDX[r] += (bdu + ((rank + 12) * U + two) * sdu) @ aA
        n = hi - lo
        dA[a] += du.T @ X[r]
        bA[a] += (bdu + (rows + 8) * U * sdu).T @ ax[r]
        dB[a] += scale * (DY[r].T @ u[r])
        bB[a] += abs(scale) * (ady[r].T @ (bu[r] + (rows + 10) * U * su))
    return (Y, bY), (u, bu), (DX, bDX), (dA, bA), (dB, bB)


def make(rows, inp, out, rank, m, dtype, atype, seed, bias=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s, std=1.0, t=F32: (torch.randn(*s, device=DEV, generator=g) * std).to(t)  # noqa: E731
    return (n(rows, inp, t=dtype), n(out, inp, std=inp ** -0.5, t=dtype), n(m, rank, inp, std=inp ** -0.5, t=atype), n(m, out, rank, t=atype),
            n(out) if bias else None, n(rows, out, t=dtype))


def segs(begin, which):
    return (torch.tensor(begin, dtype=torch.int32, device=DEV), torch.tensor(which, dtype=torch.int32, device=DEV))


def check(x, W, A, B, bias, dy, begin, which, scale=1.5, grad=True, **kw):
    sb, sa = segs(begin, which)
    (Y, bY), (u, bu), (DX, bDX), (dA, bA), (dB, bB) = reference(x, W, A, B, begin, which, scale, bias, dy)
    y, gu = ops.adapter(x, W, A, B, sb, sa, scale, bias=bias, **kw)
    within(gu, u, bu, F32, "u")
    within(y, Y, bY, x.dtype, "y")
    if not grad:
        return y, gu
    dx, gA, gB = ops.adapter_backward(x, W, A, B, gu, dy, sb, sa, scale)
    within(gA, dA, bA, F32, "dA")
    within(gB, dB, bB, F32, "dB")
    within(dx, DX, bDX, x.dtype, "dx")
    return y, gu, dx, gA, gB


TYPES = [(B16, B16), (B16, F32), (F32, F32), (F32, B16)]


@pytest.mark.parametrize("dtype,atype", TYPES)
@pytest.mark.parametrize("rows,inp,out,rank,m,begin,which", [
    (1, 1, 1, 1, 1, [0, 1], [0]),
    (1, 64, 16, 4, 2, [0, 1], [1]),
    (5, 33, 17, 3, 2, [0, 2, 2, 5], [1, 0, 0]),
    (16, 256, 100, 16, 3, [0, 4, 10, 16], [2, -1, 0]),
    (32, 264, 72, 17, 32, list(range(33)), list(range(31, -1, -1))),
    (64, 1000, 40, 64, 2, [0, 10, 50], [0, 1]),
    (65, 64, 64, 16, 2, [0, 30, 65], [0, 1]),
    (70, 63, 65, 8, 3, [3, 20, 20, 60], [0, 7, 2]),
    (128, 8, 8, 1, 1, [0, 128], [0]),
    (200, 136, 264, 32, 5, [0, 1, 2, 3, 100, 199, 200], [0, 1, 2, 3, 4, 0]),
    (257, 72, 129, 33, 2, [0, 256, 257], [1, 0]),
    (300, 520, 300, 12, 2, [0, 150, 300], [-1, 1])])
def test_adapter_and_gradients_match_the_definition(dtype, atype, rows, inp, out, rank, m, begin, which):
    check(*make(rows, inp, out, rank, m, dtype, atype, seed=rows * 13 + inp), begin, which)


@pytest.mark.parametrize("dtype,atype", TYPES)
def test_every_size_of_tile(dtype, atype):
    # 64, 128 and 256 a side, with rests in every direction
    for rows, inp, out in ((130, 72, 200), (1700, 72, 1700), (4000, 72, 3900)):
        x, W, A, B, bias, dy = make(rows, inp, out, 16, 3, dtype, atype, seed=rows, bias=rows != 1700)
        check(x, W, A, B, bias, dy, [0, rows // 3, rows // 2 + 1, rows], [2, 0, 1])


@pytest.mark.parametrize("rows,inp,out", [(1, 40, 8400), (33, 72, 9001), (64, 64, 4112), (17, 41, 8400), (5, 48, 60000)])
def test_few_rows_of_many_outputs(rows, inp, out):
    x, W, A, B, bias, dy = make(rows, inp, out, 12, 3, B16, F32, seed=rows, bias=True)
    check(x, W, A, B, bias, dy, [0, rows // 2, rows], [2, 0])


def test_tiles_that_are_not_square():
    x, W, A, B, bias, dy = make(1100, 100, 1200, 16, 3, F32, F32, seed=1100, bias=True)
    check(x, W, A, B, bias, dy, [0, 400, 777, 1100], [2, 0, 1])


@pytest.mark.parametrize("dtype", [F32, B16])
def test_long_contractions_and_many_rows_of_one_adapter(dtype):
    check(*make(1, 9000, 24, 8, 1, dtype, F32, seed=1), [0, 1], [0])
    check(*make(70, 5000, 24, 8, 1, dtype, F32, seed=2), [0, 70], [0])
    check(*make(3000, 40, 4104, 24, 1, dtype, F32, seed=3), [0, 3000], [0])


@pytest.mark.parametrize("dtype", [F32, B16])
def test_segments_of_any_kind(dtype):
    args = make(100, 48, 56, 8, 2, dtype, F32, seed=5)
    none = check(*args, [0], [])                             # no segment at all
    assert bool((none[1] == 0).all()) and bool((none[3] == 0).all()) and bool((none[4] == 0).all())
    check(*args, [-5, 40, 200], [0, 1])                      # beyond the rows on both sides
    check(*args, [0] * 50 + [100], [0] * 49 + [1])           # many empty ones
    check(*args, [0, 100], [2])                              # an adapter that does not exist
    check(*args, [0, 30, 60, 100], [1, 1, 1])                # several segments of one adapter
    few = make(20, 48, 56, 8, 2, dtype, F32, seed=6)
    check(*few, [0, 0, 0, 7, 7, 20, 20], [0, 1, 1, 0, 0, 1])
    check(*few, [4, 6], [1])


@pytest.mark.parametrize("dtype,atype", [(B16, F32), (F32, B16)])
@pytest.mark.parametrize("rows", [20, 90])
def test_strides_and_parts_of_one_array(dtype, atype, rows):
    inp, out, rank, m = 50, 38, 6, 3
    x, W, A, B, bias, dy = make(rows, inp, out, rank, m, dtype, atype, seed=rows)
    begin, which = [0, 8, rows - 3, rows], [1, 2, 0]
    y, u, dx, dA, dB = check(x, W, A, B, bias, dy, begin, which)
    sb, sa = segs(begin, which)

    def apart(t, extra):
        big = torch.full((t.shape[0] * (t.shape[1] + extra) + 1,), math.nan, device=DEV, dtype=t.dtype)[1:]
        v = big.view(t.shape[0], t.shape[1] + extra)[:, :t.shape[1]]
        v.copy_(t)
        return v
    # adapters of replicas as rows of one array, as are their gradients
    d = rank * inp + out * rank + 5
    flat = torch.full((m, d), math.nan, device=DEV, dtype=atype)
    A2, B2 = flat[:, :rank * inp].view(m, rank, inp), flat[:, rank * inp:rank * inp + out * rank].view(m, out, rank)
    A2.copy_(A)
    B2.copy_(B)
    g = torch.full((m, d), 7.0, device=DEV)
    gA, gB = g[:, :rank * inp].view(m, rank, inp), g[:, rank * inp:rank * inp + out * rank].view(m, out, rank)
    base = torch.full((rows, out + 3), 7.0, device=DEV, dtype=dtype)
    y2, u2 = ops.adapter(apart(x, 3), apart(W, 1), A2, B2, sb, sa, 1.5, bias=bias, out=base[:, :out])
    dx2, dA2, dB2 = ops.adapter_backward(apart(x, 1), apart(W, 5), A2, B2, u2, apart(dy, 1), sb, sa, 1.5, dA=gA, dB=gB,
                                         dx=torch.zeros(rows, inp + 1, device=DEV, dtype=dtype)[:, :inp])
    for p, q in ((y, y2), (u, u2), (dx, dx2), (dA, dA2), (dB, dB2)):
        assert torch.equal(p, q)
    assert bool((base[:, out:] == 7.0).all()) and bool((g[:, rank * inp + out * rank:] == 7.0).all())
    # what is not wanted
    a = ops.adapter_backward(x, W, A, B, u, dy, sb, sa, 1.5, want_adapters=False)
    b = ops.adapter_backward(x, W, A, B, u, dy, sb, sa, 1.5, want_dx=False)
    assert torch.equal(a[0], dx) and a[1] is None and b[0] is None and torch.equal(b[1], dA) and torch.equal(b[2], dB)


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("rows", [24, 100, 300])
def test_what_is_not_finite_stays_with_its_own_rows_and_adapter(dtype, rows):
    x, W, A, B, bias, dy = make(rows, 40, 48, 8, 3, dtype, F32, seed=rows)
    cut = [0, rows // 3, 2 * rows // 3, rows]
    sb, sa = segs(cut, [0, 1, 2])
    y, u = ops.adapter(x, W, A, B, sb, sa, 1.0)
    dx, dA, dB = ops.adapter_backward(x, W, A, B, u, dy, sb, sa, 1.0)
    A2, B2, x2, dy2 = A.clone(), B.clone(), x.clone(), dy.clone()
    A2[1, 3, 5], B2[1, 7, 2], B2[1, 9, 1] = math.nan, math.inf, math.nan
    lo, hi = cut[1], cut[2]
    y2, u2 = ops.adapter(x, W, A, B2, sb, sa, 1.0)
    others = torch.ones(rows, dtype=torch.bool, device=DEV)
    others[lo:hi] = False
    cols = torch.ones(48, dtype=torch.bool, device=DEV)
    cols[7] = cols[9] = False
    assert torch.equal(y2[others], y[others]) and not bool(y2[lo:hi][:, ~cols].isfinite().any())
    assert torch.allclose(y2[lo:hi][:, cols].float(), y[lo:hi][:, cols].float(), rtol=2.0 ** -7, atol=1e-5)
    y3, u3 = ops.adapter(x, W, A2, B, sb, sa, 1.0)
    assert torch.equal(y3[others], y[others]) and bool(y3[lo:hi].isnan().all())
    d3 = ops.adapter_backward(x, W, A2, B, u, dy, sb, sa, 1.0)
    assert torch.equal(d3[0][others], dx[others]) and not bool(d3[0][lo:hi, 5].isfinite().any())
    x2[lo + 1, 4], dy2[lo + 1, 4] = math.inf, math.nan
    y4, u4 = ops.adapter(x2, W, A, B, sb, sa, 1.0)
    row = torch.arange(rows, device=DEV) == lo + 1
    assert torch.equal(y4[~row], y[~row]) and not bool(y4[row].isfinite().any())
    d4 = ops.adapter_backward(x, W, A, B, u, dy2, sb, sa, 1.0)
    assert torch.equal(d4[0][~row], dx[~row]) and bool(d4[0][row].isnan().all())
    for k in (0, 2):
        assert torch.equal(d4[1][k], dA[k]) and torch.equal(d4[2][k], dB[k])
    assert not bool(d4[1][1].isfinite().any())


def test_gradient_agrees_with_differences():
    # bilinear in (A, B): in 64 bits the difference quotient of one entry is exact up to rounding; the bounds are those of the gradient
    rows, inp, out, rank, m = 9, 12, 10, 3, 2
    x, W, A, B, bias, dy = make(rows, inp, out, rank, m, F32, F32, seed=4)
    begin, which, scale = [0, 4, 9], [1, 0], 0.7
    sb, sa = segs(begin, which)
    y, u = ops.adapter(x, W, A, B, sb, sa, scale)
    dx, dA, dB = ops.adapter_backward(x, W, A, B, u, dy, sb, sa, scale)
    X, Wn, An, Bn, DY = (n64(t) for t in (x, W, A, B, dy))

    def f(X, An, Bn):
        Y = X @ Wn.T
        for s, a in enumerate(which):
            r = slice(begin[s], begin[s + 1])
            Y[r] += scale * (X[r] @ An[a].T) @ Bn[a].T
        return (Y * DY).sum()
    _, _, (DX, bDX), (_, bA), (_, bB) = reference(x, W, A, B, begin, which, scale, None, dy)
    e = 2.0 ** -10
    for which_arg, grad, bound in ((0, dx, bDX), (1, dA, bA), (2, dB, bB)):
        g = n64(grad)
        for at in list(np.ndindex(g.shape))[::3]:
            v = []
            for sgn in (e, -e):
                args = [X.copy(), An.copy(), Bn.copy()]
                args[which_arg][at] += sgn
                v.append(f(*args))
            assert abs((v[0] - v[1]) / (2 * e) - g[at]) <= bound[at] + U * abs(g[at]) + 1e-9


@pytest.mark.parametrize("rows", [12, 500])
def test_results_do_not_change_from_call_to_call_and_replays_see_new_inputs(rows):
    x, W, A, B, bias, dy = make(rows, 200, 136, 16, 2, B16, F32, seed=3)
    sb, sa = segs([0, rows // 2, rows], [0, 1])

    def both(stream=None):
        y, u = ops.adapter(x, W, A, B, sb, sa, 2.0, bias=bias, stream=stream)
        return (y, u) + ops.adapter_backward(x, W, A, B, u, dy, sb, sa, 2.0, stream=stream)
    a, b = both(), both()
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c = both(s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(p, q) for p, q in zip(a, c))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for n in range(3):
        x.copy_(torch.randn(rows, 200, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, both()))


def test_refusals():
    x, W, A, B, bias, dy = make(10, 16, 24, 4, 2, F32, F32, seed=0)
    sb, sa = segs([0, 4, 10], [0, 1])
    y, u = ops.adapter(x, W, A, B, sb, sa, 1.0)
    for bad in (dict(x=x[0]), dict(x=x.half()), dict(W=W.bfloat16()), dict(W=W[:, :8]), dict(A=A[:, :, :8]), dict(B=B[:1]), dict(B=B.bfloat16()),
                dict(seg_begin=sb[:2]), dict(seg_begin=sb.long()), dict(seg_adapter=sa.long()), dict(bias=bias[:3]), dict(bias=bias.bfloat16()),
                dict(out=y[:, :8]), dict(out=y.bfloat16()), dict(x=x.cpu()), dict(W=W.t().contiguous().t()),
                dict(A=torch.zeros(2, 65, 16, device=DEV), B=torch.zeros(2, 24, 65, device=DEV)),
                dict(A=torch.zeros(2, 0, 16, device=DEV), B=torch.zeros(2, 24, 0, device=DEV))):
        kw = dict(dict(x=x, W=W, A=A, B=B, seg_begin=sb, seg_adapter=sa, scale=1.0), **bad)
        with pytest.raises(lsam.LsamError) as e:
            ops.adapter(**kw)
        assert e.value.code == lsam.EINVAL
    for bad in (dict(u=u[:, :2]), dict(u=u.bfloat16()), dict(dy=dy[:, :8]), dict(dx=x), dict(dx=dy[:, :16]), dict(dA=A[:1]), dict(dB=B),
                dict(dA=A.bfloat16())):
        kw = dict(dict(x=x, W=W, A=A, B=B, u=u, dy=dy, seg_begin=sb, seg_adapter=sa, scale=1.0), **bad)
        with pytest.raises(lsam.LsamError) as e:
            ops.adapter_backward(**kw)
        assert e.value.code == lsam.EINVAL
    square = torch.zeros(10, 16, device=DEV)
    with pytest.raises(lsam.LsamError) as e:
        ops.adapter(square, torch.zeros(16, 16, device=DEV), A, torch.zeros(2, 16, 4, device=DEV), sb, sa, 1.0, out=square)
    assert "lies over" in str(e.value)
    none = ops.adapter(torch.zeros(0, 16, device=DEV), W, A, B, *segs([0], []), 1.0)
    assert none[0].shape == (0, 24)
    z = ops.adapter_backward(torch.zeros(0, 16, device=DEV), W, A, B, none[1], torch.zeros(0, 24, device=DEV), *segs([0], []), 1.0)
    assert bool((z[1] == 0).all()) and bool((z[2] == 0).all())


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("rank", [33, 64])
def test_large_ranks_of_many_rows(dtype, rank):
    x, W, A, B, bias, dy = make(7300, 136, 72, rank, 2, dtype, dtype, seed=rank, bias=True)
    check(x, W, A, B, bias, dy, [0, 3000, 3001, 7290], [1, 0, 1])


@pytest.mark.parametrize("dtype", [F32, B16])
def test_more_segments_than_lanes(dtype):
    rows, n = 300, 620                                       # every second one empty: 128 in a tile of 64 rows
    begin = [min(rows, i // 2) for i in range(n + 1)]
    x, W, A, B, bias, dy = make(rows, 72, 104, 8, 7, dtype, F32, seed=n, bias=True)
    check(x, W, A, B, bias, dy, begin, [i % 8 - 1 for i in range(n)])
