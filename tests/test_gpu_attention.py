"""lsam_attention and its gradient against the definition in 64 bits.

Tolerances (u = 2^-24; r = 2^-8 for bfloat16, 0 for fp32).  A score is a sum of dim products, in any order: (dim + 8) u of scale sum |q k|.  Its
exponent adds 4 u of itself, and lse is off by as much as the worst score of its row, by the n additions and one power of its sum, and by a logarithm and two
products (4 u of itself and 4 u): so p is off by e_p = the sum of both and 8 u, of itself.  o: p rounded by r, n additions.  The gradient's d_o v is a sum of dim products,
d_o o one more with the o that was stored; ds adds the errors of its factors, and r for its own rounding; sums over n rows add n u of absolute values.
What is stored in bfloat16 is rounded by r of itself."""
import math

import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, B16 = torch.float32, torch.bfloat16


def reference(q, k, v, do, scale, dtype):
    """One sequence, [n, heads, dim]: {name: (value, bound)}."""
    q, k, v, do = (t.double().transpose(0, 1) for t in (q, k, v, do))
    H, n, dim = q.shape
    group = H // k.shape[0]
    r = 2.0 ** -8 if dtype == B16 else 0.0
    K, V = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    T = lambda t: t.transpose(1, 2)  # noqa: E731
    later = torch.ones(n, n, device=DEV, dtype=torch.bool).triu(1)
    s = (scale * q @ T(K)).masked_fill(later, -math.inf)
    size = (scale * q.abs() @ T(K.abs())).masked_fill(later, 0)
    lse = torch.logsumexp(s, 2, keepdim=True)
    p = torch.exp(s - lse)
    es = (dim + 8) * U * size + 4 * U * s.masked_fill(later, 0).abs()
    el = es.amax(2, keepdim=True) + (n + 10) * U + 4 * U * lse.abs()
    ep = torch.expm1(es + el) + 8 * U
    o = p @ V
    eo = (p * (r + ep)) @ V.abs() + (n + 8) * U * (p @ V.abs())
    eo_stored = eo + (r + U) * (o.abs() + eo)
    dp, delta = do @ T(V), (do * o).sum(2, keepdim=True)
    edp = (dim + 8) * U * (do.abs() @ T(V.abs()))
    edelta = (do.abs() * eo_stored).sum(2, keepdim=True) + (dim + 8) * U * (do * o).abs().sum(2, keepdim=True)
    ds = p * (dp - delta)
    gap = (dp - delta).abs()
    eds = p * (1 + ep) * (edp + edelta + 2 * U * (dp.abs() + delta.abs())) + ep * p * gap
    eds = eds + (r + U) * (p * gap + eds)
    fold = lambda t: t.reshape(-1, group, n, dim).sum(1)  # noqa: E731
    out = dict(o=(o, eo), lse=(lse[:, :, 0], el[:, :, 0]))
    out["dq"] = (scale * ds @ K, scale * (eds @ K.abs() + (n + 8) * U * (ds.abs() @ K.abs())))
    out["dk"] = (fold(scale * T(ds) @ q), fold(scale * (T(eds) @ q.abs() + (group * n + 8) * U * (T(ds.abs()) @ q.abs()))))
    pv = p * (r + ep + (group * n + 8) * U)
    out["dv"] = (fold(T(p) @ do), fold(T(pv) @ do.abs()))
    return {name: tuple(t if name == "lse" else t.transpose(0, 1) for t in pair) for name, pair in out.items()}


def near(got, want, bound, what):
    bound = bound + (2.0 ** -8 * (want.abs() + bound) if got.dtype == B16 else U * want.abs()) + 1e-37
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (what, float((off / bound).max()))


def check(q, k, v, do, offsets, scale=None, floor=0.0):
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    r = ops.attention(q, k, v, off, scale=scale, save=True)
    grads = ops.attention_backward(q, k, v, off, r.o, r.lse, do, scale=scale)
    got = dict(o=r.o, lse=r.lse, dq=grads[0], dk=grads[1], dv=grads[2])
    rows = q.shape[0]
    for lo, hi in zip(offsets, offsets[1:]):
        lo, hi = max(lo, 0), min(hi, rows)
        if lo >= hi:
            continue
        want = reference(q[lo:hi], k[lo:hi], v[lo:hi], do[lo:hi], q.shape[2] ** -0.5 if scale is None else scale, q.dtype)
        for name, (value, bound) in want.items():
            near(got[name][:, lo:hi] if name == "lse" else got[name][lo:hi], value, bound + floor, name)
    return got


def make(rows, H, KV, dim, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda h: (torch.randn(rows, h, dim, device=DEV, generator=g) * std).to(dtype)  # noqa: E731
    return n(H), n(KV), n(KV), n(H)


TYPES = pytest.mark.parametrize("dtype", [F32, B16])


@TYPES
@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 64, 65, 127, 128, 129, 200, 321])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_sequence(rows, dim, dtype):
    check(*make(rows, 2, 1, dim, dtype, seed=rows + dim), [0, rows])


@TYPES
@pytest.mark.parametrize("dim", [1, 3, 8, 31, 33, 40, 63, 65, 72, 100, 120, 127])
def test_other_widths(dim, dtype):
    check(*make(150, 2, 2, dim, dtype, seed=dim), [0, 70, 150])


@TYPES
@pytest.mark.parametrize("H,KV", [(1, 1), (3, 1), (8, 8), (6, 3), (16, 16), (24, 8), (10, 5), (12, 4), (40, 8), (7, 7)])
def test_heads_and_groups(H, KV, dtype):
    check(*make(140, H, KV, 32, dtype, seed=H), [0, 3, 140])


@TYPES
@pytest.mark.parametrize("offsets", [[0, 0, 1, 1, 2, 300], [0, 64, 128, 192, 300], list(range(301)), [0, 1, 299, 300], [0, 127, 129, 255, 257, 300],
                                     [0, 31, 33, 63, 65, 95, 97, 300], [0] * 70 + [150] * 70 + [300]])
def test_packed_sequences(offsets, dtype):
    check(*make(300, 4, 2, 64, dtype, seed=len(offsets)), offsets)


@TYPES
@pytest.mark.parametrize("offsets", [[5, 70, 71, 290], [140, 150], [0, 30], [299, 300], [50, 50, 50]])
def test_rows_of_no_sequence_are_not_looked_at_and_not_written(offsets, dtype):
    q, k, v, do = make(300, 4, 2, 40, dtype, seed=offsets[0])
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    inside = slice(offsets[0], offsets[-1])
    clean = ops.attention(q, k, v, off, save=True)
    for t in (q, k, v, do):
        t[:offsets[0]] = math.nan
        t[offsets[-1]:] = math.nan
    check(q, k, v, do, offsets)
    outs = [torch.full_like(t, 7.0) for t in (q, q, k, v)]
    r = ops.attention(q, k, v, off, save=True, out=outs[0])
    assert torch.equal(r.o[inside], clean.o[inside])
    ops.attention_backward(q, k, v, off, r.o, r.lse, do, dq=outs[1], dk=outs[2], dv=outs[3])
    for t in outs:
        assert bool((t[:offsets[0]] == 7).all()) and bool((t[offsets[-1]:] == 7).all()) and bool(t[inside].isfinite().all())


@TYPES
def test_offsets_outside_the_rows_are_taken_as_the_nearest_inside(dtype):
    q, k, v, do = make(100, 2, 1, 64, dtype, seed=1)
    a, b = check(q, k, v, do, [-5, 30, 200]), check(q, k, v, do, [0, 30, 100])
    assert all(torch.equal(a[n], b[n]) for n in a)


@TYPES
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 100])
def test_what_is_not_finite_reaches_only_rows_that_see_it(value, dim, dtype):
    """Row 100 of one sequence of three: keys and values reach rows 100 .. 159 of it, queries only their own row, d_o the rows up to 100."""
    offsets, bad = [0, 60, 160, 230], 100
    q, k, v, do = make(230, 2, 1, dim, dtype, seed=dim)
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    clean = ops.attention(q, k, v, off, save=True)
    grads = ops.attention_backward(q, k, v, off, clean.o, clean.lse, do)
    rows = torch.arange(230, device=DEV)
    other = (rows < 60) | (rows >= 160)
    for which in range(3):
        part = [t.clone() for t in (q, k, v)]
        part[which][bad, :, 3] = value
        r = ops.attention(*part, off, save=True)
        safe = rows != bad if which == 0 else other | (rows < bad)
        assert torch.equal(r.o[safe], clean.o[safe]) and torch.equal(r.lse[:, safe], clean.lse[:, safe]), which
        if which == 2 or math.isnan(value):                           # an infinite score may be -inf, which weighs nothing
            assert not bool(r.o[bad].isfinite().all())
        # o and lse of the clean call: what the bad row alone does to the gradients
        dq, dk, dv = ops.attention_backward(*part, off, clean.o, clean.lse, do)
        if which == 0:                                            # a query: its own dq, and dk, dv of rows up to it
            assert torch.equal(dq[safe], grads[0][safe])
            seen = other | (rows > bad)
            assert torch.equal(dk[seen], grads[1][seen]) and torch.equal(dv[seen], grads[2][seen])
        else:                                                     # a key or value: dq of rows from it on, its own dk, dv
            seen = other | (rows < bad)
            assert torch.equal(dq[seen], grads[0][seen])
            alone = rows != bad
            assert torch.equal(dk[alone], grads[1][alone]) and torch.equal(dv[alone], grads[2][alone])
    g = do.clone()
    g[bad, :, 3] = value
    dq, dk, dv = ops.attention_backward(q, k, v, off, clean.o, clean.lse, g)
    alone, seen = rows != bad, other | (rows > bad)
    assert torch.equal(dq[alone], grads[0][alone]) and torch.equal(dk[seen], grads[1][seen]) and torch.equal(dv[seen], grads[2][seen])


@TYPES
@pytest.mark.parametrize("scale", [0.0, 1e-3, 1.0, 30.0])
def test_scales_up_to_one_key_that_takes_all(scale, dtype):
    q, k, v, do = make(150, 2, 1, 64, dtype, seed=3)
    check(q, k, v, do, [0, 150], scale=scale)


@TYPES
def test_scores_far_from_zero(dtype):
    """Maxima that grow, and fall, from tile to tile by far more than a power of two can hold."""
    q, k, v, do = make(260, 1, 1, 32, dtype, seed=4)
    q.fill_(1.0)
    k.zero_()
    k[:, 0, 0] = (torch.arange(260, device=DEV) // 64 % 2).to(dtype) * 500 - 250
    check(q, k, v, do, [0, 260], scale=1.0)


@TYPES
@pytest.mark.parametrize("dim", [64, 36])
def test_parts_of_one_array_and_heads_outside_of_rows(dim, dtype):
    rows, H, KV, offsets = 170, 4, 2, [0, 100, 170]
    q, k, v, do = make(rows, H, KV, dim, dtype, seed=5)
    want = check(q, k, v, do, offsets)
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)

    def compare(lay):
        qkv, grads, o, g = lay(H + 2 * KV), lay(H + 2 * KV), lay(H), lay(H)
        qs, ks, vs = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
        for a, b in ((qs, q), (ks, k), (vs, v), (g, do)):
            a.copy_(b)
        lse = ops.attention(qs, ks, vs, off, save=True, out=o).lse
        got = ops.attention_backward(qs, ks, vs, off, o, lse, g, dq=grads[:, :H], dk=grads[:, H:H + KV], dv=grads[:, H + KV:])
        assert torch.equal(o, want["o"]) and torch.equal(lse, want["lse"])
        assert all(torch.equal(a, want[n]) for a, n in zip(got, ("dq", "dk", "dv")))
    compare(lambda h: torch.zeros(rows, h, dim, dtype=dtype, device=DEV))
    compare(lambda h: torch.zeros(h, rows, dim, dtype=dtype, device=DEV).transpose(0, 1))
    compare(lambda h: torch.zeros(rows + 1, h, dim + 3, dtype=dtype, device=DEV)[1:, :, 1:1 + dim])         # no row aligned to 16 bytes


def test_the_formula_against_differences():
    q, k, v, do = (t.double() for t in make(5, 2, 1, 3, F32, seed=6))
    want = reference(q, k, v, do, 0.7, F32)

    def value(*t):
        return (reference(*t, do, 0.7, F32)["o"][0] * do).sum()
    for i, (t, name) in enumerate(((q, "dq"), (k, "dk"), (v, "dv"))):
        for n in range(t.numel()):
            step = torch.zeros_like(t).view(-1)
            step[n] = 1e-5
            ends = []
            for sign in (1, -1):
                args = [q, k, v]
                args[i] = t + sign * step.view_as(t)
                ends.append(value(*args))
            assert abs(float((ends[0] - ends[1]) / 2e-5 - want[name][0].reshape(-1)[n])) < 1e-7


@TYPES
def test_the_same_call_gives_the_same_bits(dtype):
    q, k, v, do = make(700, 6, 2, 80, dtype, seed=7)
    off = torch.tensor([0, 300, 301, 700], dtype=torch.int64, device=DEV)
    r = ops.attention(q, k, v, off, save=True)
    first = ops.attention_backward(q, k, v, off, r.o, r.lse, do)
    for _ in range(3):
        again = ops.attention(q, k, v, off, save=True)
        assert torch.equal(again.o, r.o) and torch.equal(again.lse, r.lse)
        assert all(torch.equal(a, b) for a, b in zip(first, ops.attention_backward(q, k, v, off, r.o, r.lse, do)))
    assert ops.attention(q, k, v, off).lse is None


def test_no_rows_and_no_sequences():
    e = torch.empty(0, 2, 8, device=DEV)
    off = torch.zeros(3, dtype=torch.int64, device=DEV)
    r = ops.attention(e, e, e, off, save=True)
    assert r.o.shape == (0, 2, 8) and all(t.shape == (0, 2, 8) for t in ops.attention_backward(e, e, e, off, r.o, r.lse, e))
    x = torch.ones(4, 2, 8, device=DEV)
    out = torch.full_like(x, 3.0)
    ops.attention(x, x, x, off[:1], out=out)
    assert bool((out == 3).all())


def test_refusals():
    q, k, v, do = make(10, 4, 2, 16, F32, seed=8)
    off = torch.tensor([0, 10], dtype=torch.int64, device=DEV)
    r = ops.attention(q, k, v, off, save=True)
    wide = torch.zeros(10, 4, 136, device=DEV)
    for call, word in [(lambda: ops.attention(q[0], k, v, off), "indices"), (lambda: ops.attention(q, k[:5], v, off), "shape"),
                       (lambda: ops.attention(q, k, v.to(B16), off), "float32"), (lambda: ops.attention(q, k, v, off.int()), "int64"),
                       (lambda: ops.attention(q[:, :3], k, v, off), "multiple"), (lambda: ops.attention(wide, wide, wide, off), "dim"),
                       (lambda: ops.attention(q, k, v, off, scale=-1.0), "scale"), (lambda: ops.attention(q, k, v, off, scale=math.nan), "scale"),
                       (lambda: ops.attention(q, k, v, off, scale=math.inf), "scale"), (lambda: ops.attention(q, k, v, off, out=q), "lies over"),
                       (lambda: ops.attention_backward(q, k, v, off, r.o, r.lse[:, :5], do), "shape"),
                       (lambda: ops.attention_backward(q, k, v, off, r.o, r.lse, do, dk=v), "lies over"),
                       (lambda: ops.attention_backward(q, k, v, off, r.o, r.lse, do, dq=do), "lies over"),
                       (lambda: ops.attention(q.half(), k.half(), v.half(), off), "bfloat16"),
                       (lambda: ops.attention(q.requires_grad_(), k, v, off), "gradient")]:
        with pytest.raises(lsam.LsamError) as e:
            call()
        assert e.value.code == lsam.EINVAL and word in str(e.value), (word, str(e.value))
