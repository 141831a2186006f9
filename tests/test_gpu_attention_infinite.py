"""Scores of -inf weigh nothing, whatever made them: an infinite key, or a product that passes the range of fp32.  A call with such a key gives the bits of one
whose key is finite and so far below the others that its weight is 0.  A value that is infinite is so in the result, and only there."""
import math

import pytest
import torch

from paper_2509_03110_amd import ops

from test_gpu_attention import B16, DEV, F32, TYPES, make  # noqa: E402

pytestmark = pytest.mark.gpu
# rows and heads shared; rows, or keys, of a wavefront's own; that with shared heads.  Whole units of eight numbers, and others
FORMS = pytest.mark.parametrize("rows,H,KV,dim", [(230, 2, 1, 64), (230, 4, 2, 100), (200, 2, 2, 128), (520, 52, 52, 64), (520, 52, 52, 35), (1000, 80, 40, 32)])


def same(a, b, what):
    assert torch.equal(a, b), (what, float((a != b).float().mean()))


def compare(q, k, v, do, offsets, far, infinite, bad, dtype):
    """`far`, `infinite`: what stands in number 3 of key `bad` in both calls."""
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    got = []
    for value in (far, infinite):
        keys = k.clone()
        keys[bad, :, 3] = value
        r = ops.attention(q, keys, v, off, save=True)
        got.append((r.o, r.lse) + ops.attention_backward(q, keys, v, off, r.o, r.lse, do))
    (o, lse, dq, dk, dv), (o2, lse2, dq2, dk2, dv2) = got
    assert bool(o.isfinite().all()) and bool((dv[bad] == 0).all()) and bool((dk[bad] == 0).all())
    same(o2, o, "o")
    same(lse2, lse, "lse")
    same(dk2, dk, "dk")
    same(dv2, dv, "dv")
    others = [i for i in range(q.shape[2]) if i != 3]                            # 0 times what is not finite is in the sum of number 3
    same(dq2[:, :, others], dq[:, :, others], "dq")
    if math.isfinite(infinite):
        same(dq2, dq, "dq")


@TYPES
@FORMS
def test_infinite_keys(rows, H, KV, dim, dtype):
    q, k, v, do = make(rows, H, KV, dim, dtype, seed=rows + dim)
    q[:, :, 3] = q[:, :, 3].abs() + 0.1
    compare(q, k, v, do, [0, 60, 70, rows], -1e30, -math.inf, 100, dtype)
    compare(-q, k, v, do, [0, 60, 70, rows], 1e30, math.inf, 150, dtype)


@FORMS
def test_products_past_the_range_of_fp32(rows, H, KV, dim):
    q, k, v, do = make(rows, H, KV, dim, F32, seed=rows + dim)
    q[:, :, 3], k[:, :, 3] = 1.0123e25, 0.0
    for infinite in (-1.077e25, -3.3e38, -1.0039e25):
        compare(q, k, v, do, [0, 60, 70, rows], -1e3, infinite, 100, F32)


@TYPES
def test_a_row_whose_scores_are_all_infinite_and_one_of_nan(dtype):
    q, k, v, do = make(300, 2, 1, 64, dtype, seed=1)
    q[:, :, 3] = 1.0
    off = torch.tensor([0, 100, 300], dtype=torch.int64, device=DEV)
    want = ops.attention(q, k, v, off, save=True)
    k[100, :, 3], k[200, :, 7] = -math.inf, math.nan
    r = ops.attention(q, k, v, off, save=True)
    assert bool(r.o[100].isnan().all()) and bool(r.o[200:].isnan().all()) and bool(r.o[101:200].isfinite().all())
    same(r.o[:100], want.o[:100], "o")


# one token: columns shared by wavefronts, or each with columns of its own (of the prefix); one part, or many
STEPS = pytest.mark.parametrize("S,H,KV,dim,cap,prefix", [(1, 4, 2, 64, 90, 0), (3, 4, 2, 100, 700, 300), (40, 8, 1, 128, 50, 1000), (70, 8, 8, 64, 40, 300), (2, 40, 1, 36, 200, 0)])


def caches(S, H, KV, dim, cap, prefix, dtype):
    g = torch.Generator(device=DEV).manual_seed(S + dim)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g).to(dtype)  # noqa: E731
    q = n(S, H, dim)
    q[:, :, 3] = q[:, :, 3].abs() + 0.1
    c = dict(q=q, k=n(S, cap, KV, dim), v=n(S, cap, KV, dim), lengths=torch.full((S,), cap - 5, dtype=torch.int32, device=DEV))
    if prefix:
        c.update(prefix_k=n(prefix, KV, dim), prefix_v=n(prefix, KV, dim))
    return c


def rows_of(c, name):
    """Key or value 20 of the prefix, or of each cache but the first."""
    return c[name][20] if name.startswith("prefix") else c[name][min(1, c[name].shape[0] - 1):, 20]


@TYPES
@STEPS
def test_one_tokens_infinite_keys(S, H, KV, dim, cap, prefix, dtype):
    for name in ("k", "prefix_k")[:2 if prefix else 1]:
        got = []
        for value in (-1e30, -math.inf):
            c = caches(S, H, KV, dim, cap, prefix, dtype)
            rows_of(c, name)[..., 3] = value
            got.append(ops.attention_step(**c))
        assert bool(got[0].isfinite().all())
        same(got[1], got[0], name)


@STEPS
def test_one_tokens_products_past_the_range_of_fp32(S, H, KV, dim, cap, prefix):
    got = []
    for value in (-1e3, -1.077e25):
        c = caches(S, H, KV, dim, cap, prefix, F32)
        for name in ("q", "k", "prefix_k")[:3 if prefix else 2]:
            c[name][..., 3] = 1.0123e25 if name == "q" else 0.0
        rows_of(c, "k")[..., 3] = value
        got.append(ops.attention_step(**c))
    assert bool(got[0].isfinite().all())
    same(got[1], got[0], "o")


@TYPES
@STEPS
def test_one_tokens_infinite_values(S, H, KV, dim, cap, prefix, dtype):
    others = [i for i in range(dim) if i != 3]
    for name in ("v", "prefix_v")[:2 if prefix else 1]:
        c = caches(S, H, KV, dim, cap, prefix, dtype)
        clean = ops.attention_step(**c)
        rows_of(c, name)[..., 3] = -math.inf
        got = ops.attention_step(**c)
        first = 0 if name == "prefix_v" else min(1, S - 1)
        assert bool((got[first:, :, 3] == -math.inf).all())
        same(got[:, :, others], clean[:, :, others], name)
        same(got[:first], clean[:first], name)
    c = caches(S, H, KV, dim, cap, prefix, dtype)
    c["v"][:, 7, :, 5] = math.nan
    assert bool(ops.attention_step(**c)[:, :, 5].isnan().all())


@TYPES
def test_one_token_that_meets_only_scores_of_minus_infinity(dtype):
    c = caches(3, 4, 2, 64, 90, 0, dtype)
    c["k"][..., 3] = -math.inf
    assert bool((ops.attention_step(**c) == 0).all())


@TYPES
def test_places_behind_the_length_that_share_memory_with_those_before(dtype):
    """Strides below the width: what lies behind a sequence's last place is part of places that it has, infinite ones among them, and still weighs nothing."""
    S, H, KV, dim, cap, n = 3, 4, 2, 64, 60, 37
    g = torch.Generator(device=DEV).manual_seed(11)
    q = torch.randn(S, H, dim, device=DEV, generator=g).to(dtype)
    lengths = torch.full((S,), n, dtype=torch.int32, device=DEV)
    for step in (0, 8, 32):
        base = torch.randn(2, S, KV, 2048 + dim, device=DEV, generator=g).to(dtype)
        base[1, :, :, (n - 1) * step + dim - 1] = math.inf                      # the last number of the last place
        k, v = (t.as_strided((S, cap, KV, dim), (KV * (2048 + dim), step, 2048 + dim, 1), t.storage_offset()) for t in base)
        got = ops.attention_step(q, k, v, lengths)
        same(got, ops.attention_step(q, k.contiguous(), v.contiguous(), lengths), step)
        assert bool((got[..., -1] == math.inf).all()) and bool(got[..., :dim - max(step, 1)].isfinite().all())
        prefix = ops.attention_step(q, k[:, :0], v[:, :0], lengths, prefix_k=k[0, :n], prefix_v=v[0, :n])
        same(prefix, ops.attention_step(q, k[:, :0], v[:, :0], lengths, prefix_k=k[0, :n].contiguous(), prefix_v=v[0, :n].contiguous()), step)
