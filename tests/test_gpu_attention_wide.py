"""lsam_attention and its gradient where rows and heads fill the chip and each wavefront has rows, or keys, of its own; the reference and the
tolerances are those of test_gpu_attention."""
import math

import pytest
import torch

from paper_2509_03110_amd import ops

import test_gpu_attention as few  # noqa: E402
from test_gpu_attention import DEV, TYPES, check, make  # noqa: E402

pytestmark = pytest.mark.gpu


@TYPES
@pytest.mark.parametrize("dim", [1, 8, 31, 33, 64, 72, 96, 100, 127, 128])
def test_widths(dim, dtype):
    check(*make(530, 52, 52, dim, dtype, seed=dim), [0, 5, 300, 530])


@TYPES
@pytest.mark.parametrize("H,KV,rows", [(64, 16, 520), (64, 64, 513), (256, 8, 130), (300, 100, 129), (257, 257, 1), (256, 256, 128), (86, 43, 1200)])
def test_heads_and_groups(H, KV, rows, dtype):
    check(*make(rows, H, KV, 16, dtype, seed=H), [0, min(3, rows), rows])


@TYPES
@pytest.mark.parametrize("offsets", [[0, 0, 1, 1, 2, 640], list(range(71)) + [300, 640], [0, 127, 129, 255, 257, 640], [0, 1, 639, 640],
                                     [0] * 70 + [150] * 70 + [640], [0, 128, 256, 384, 512, 640], [0, 95, 97, 159, 161, 640]])
def test_packed_sequences(offsets, dtype):
    check(*make(640, 52, 52, 32, dtype, seed=len(offsets)), offsets)


@TYPES
@pytest.mark.parametrize("offsets", [[5, 70, 71, 630], [140, 150], [0, 30], [639, 640], [300, 300], [129, 256]])
def test_rows_of_no_sequence_are_not_looked_at_and_not_written(offsets, dtype):
    q, k, v, do = make(640, 52, 52, 40, dtype, seed=offsets[0])
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
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dim", [64, 100])
def test_what_is_not_finite_reaches_only_rows_that_see_it(value, dim, dtype):
    """Row 300 of one sequence of three, in some heads only."""
    offsets, bad, H = [0, 200, 420, 520], 300, 52
    q, k, v, do = make(520, H, H, dim, dtype, seed=dim)
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    clean = ops.attention(q, k, v, off, save=True)
    grads = ops.attention_backward(q, k, v, off, clean.o, clean.lse, do)
    rows = torch.arange(520, device=DEV)
    other = (rows < 200) | (rows >= 420)
    heads, rest = slice(0, H, 3), torch.arange(H, device=DEV) % 3 != 0
    for which in range(3):
        part = [t.clone() for t in (q, k, v)]
        part[which][bad, heads, 3] = value
        r = ops.attention(*part, off, save=True)
        safe = rows != bad if which == 0 else other | (rows < bad)
        assert torch.equal(r.o[safe], clean.o[safe]) and torch.equal(r.lse[:, safe], clean.lse[:, safe]), which
        assert torch.equal(r.o[:, rest], clean.o[:, rest])
        if which == 2 or math.isnan(value):
            assert not bool(r.o[bad, 0].isfinite().all())
        dq, dk, dv = ops.attention_backward(*part, off, clean.o, clean.lse, do)
        assert all(torch.equal(a[:, rest], b[:, rest]) for a, b in zip((dq, dk, dv), grads))
        if which == 0:
            seen = other | (rows > bad)
            assert torch.equal(dq[safe], grads[0][safe]) and torch.equal(dk[seen], grads[1][seen]) and torch.equal(dv[seen], grads[2][seen])
        else:
            seen, alone = other | (rows < bad), rows != bad
            assert torch.equal(dq[seen], grads[0][seen]) and torch.equal(dk[alone], grads[1][alone]) and torch.equal(dv[alone], grads[2][alone])
    g = do.clone()
    g[bad, heads, 3] = value
    dq, dk, dv = ops.attention_backward(q, k, v, off, clean.o, clean.lse, g)
    alone, seen = rows != bad, other | (rows > bad)
    assert torch.equal(dq[alone], grads[0][alone]) and torch.equal(dk[seen], grads[1][seen]) and torch.equal(dv[seen], grads[2][seen])


@TYPES
@pytest.mark.parametrize("scale", [0.0, 1e-3, 1.0, 30.0])
def test_scales_up_to_one_key_that_takes_all(scale, dtype):
    """A weight below 2^-126, fp32's smallest normal number, counts as 0, and so does its ds.  A key that has only such weights misses up to
    2^-126 scale |d_o v - d_o o| |q| a row in dk (seen at scale 30: all of 3.5e-35); no |d_o v| is above |d_o| |v|, nor |d_o o|, a mean of such."""
    q, k, v, do = make(520, 52, 52, 64, dtype, seed=3)
    most = lambda t: float(t.float().norm(dim=2).max())  # noqa: E731
    check(q, k, v, do, [0, 520], scale=scale, floor=2.0 ** -126 * scale * 520 * 2 * most(do) * most(v) * most(q))


@TYPES
def test_scores_far_from_zero(dtype):
    q, k, v, do = make(520, 52, 52, 32, dtype, seed=4)
    q.fill_(1.0)
    k.zero_()
    k[:, :, 0] = (torch.arange(520, device=DEV)[:, None] // 64 % 2).to(dtype) * 500 - 250
    check(q, k, v, do, [0, 520], scale=1.0)


@TYPES
@pytest.mark.parametrize("dim", [64, 36])
def test_parts_of_one_array_and_heads_outside_of_rows(dim, dtype):
    rows, H, KV, offsets = 530, 104, 52, [0, 100, 530]
    q, k, v, do = make(rows, H, KV, dim, dtype, seed=5)
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    want = check(q, k, v, do, offsets)

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
    compare(lambda h: torch.zeros(rows + 1, h, dim + 3, dtype=dtype, device=DEV)[1:, :, 1:1 + dim])


@TYPES
def test_the_same_call_gives_the_same_bits(dtype):
    q, k, v, do = make(900, 64, 64, 80, dtype, seed=7)
    off = torch.tensor([0, 300, 301, 900], dtype=torch.int64, device=DEV)
    r = ops.attention(q, k, v, off, save=True)
    first = ops.attention_backward(q, k, v, off, r.o, r.lse, do)
    for _ in range(3):
        again = ops.attention(q, k, v, off, save=True)
        assert torch.equal(again.o, r.o) and torch.equal(again.lse, r.lse)
        assert all(torch.equal(a, b) for a, b in zip(first, ops.attention_backward(q, k, v, off, r.o, r.lse, do)))


@TYPES
def test_one_long_sequence(dtype):
    """A row of 4099 keys, the first rows and a tile in the middle against the reference, which does not hold all scores at once."""
    q, k, v, do = make(4099, 8, 2, 64, dtype, seed=9)
    off = torch.tensor([0, 4099], dtype=torch.int64, device=DEV)
    r = ops.attention(q, k, v, off, save=True)
    for lo in (0, 1000, 2040, 4000):
        n = min(lo + 99, 4099)
        want = few.reference(q[:n, :4], k[:n, :1], v[:n, :1], do[:n, :4], 64 ** -0.5, dtype)
        few.near(r.o[lo:n, :4], want["o"][0][lo:], want["o"][1][lo:], "o")
        few.near(r.lse[:4, lo:n], want["lse"][0][:, lo:], want["lse"][1][:, lo:], "lse")
