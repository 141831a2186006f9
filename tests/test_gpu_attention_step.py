"""lsam_attention_step against the definition in 64 bits.

Tolerances (u = 2^-24; r = 2^-8 for bfloat16, 0 for fp32): a score is a sum of dim products, (dim + 8) u of scale sum |q k|, and its exponent adds
4 u of itself; a weight is off by its own and by the worst of its row's, by n + 40 additions of the sum, and by the powers that join parts: 20 u.
Values are weighted with weights rounded by r, in n + 80 additions; what is stored in bfloat16 is rounded by r of itself."""
import math

import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, B16 = torch.float32, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F32, B16])


def check(o, q, k, v, lengths, pk, pv, scale):
    S, H, dim = q.shape
    group = H // k.shape[2]
    r = 2.0 ** -8 if q.dtype == B16 else 0.0
    for s in range(S):
        n = min(max(int(lengths[s]), 0), k.shape[1])
        K = torch.cat(([] if pk is None else [pk]) + [k[s, :n]]).double().repeat_interleave(group, 1)      # [n, H, dim]
        V = torch.cat(([] if pv is None else [pv]) + [v[s, :n]]).double().repeat_interleave(group, 1)
        if K.shape[0] == 0:
            assert bool((o[s] == 0).all())
            continue
        z, size = scale * (K * q[s].double()).sum(2), scale * (K * q[s].double()).abs().sum(2)
        p = torch.softmax(z, 0)
        e = (dim + 8) * U * size + 4 * U * z.abs()
        ep = torch.expm1(e + e.amax(0)) + (K.shape[0] + 60) * U + r
        want, bound = (p[:, :, None] * V).sum(0), ((p * (ep + (K.shape[0] + 80) * U))[:, :, None] * V.abs()).sum(0)
        bound = bound + (r + U) * (want.abs() + bound) + 1e-37
        off = (o[s].double() - want).abs()
        assert bool((off <= bound).all()), (s, float((off / bound).max()))


def make(S, H, KV, dim, cap, prefix, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g).to(dtype)  # noqa: E731
    lengths = torch.randint(0, cap + 1, (S,), device=DEV, generator=g, dtype=torch.int32)
    if S > 2:
        lengths[0], lengths[1], lengths[2] = 0, min(1, cap), cap
    return dict(q=n(S, H, dim), k=n(S, cap, KV, dim), v=n(S, cap, KV, dim), lengths=lengths,
                prefix_k=n(prefix, KV, dim) if prefix is not None else None, prefix_v=n(prefix, KV, dim) if prefix is not None else None)


def run(c, scale=None):
    o = ops.attention_step(**c, scale=scale)
    check(o, c["q"], c["k"], c["v"], c["lengths"], c["prefix_k"], c["prefix_v"], c["q"].shape[2] ** -0.5 if scale is None else scale)
    return o


@TYPES
@pytest.mark.parametrize("S,H,KV,dim,cap,prefix", [
    (1, 1, 1, 64, 1, None), (1, 8, 2, 128, 1000, None), (3, 4, 4, 64, 127, None), (5, 6, 3, 72, 129, 1), (4, 8, 8, 128, 33, 31),
    (3, 66, 2, 32, 200, 65), (33, 4, 2, 64, 40, 300), (40, 8, 1, 100, 5, 1000), (2, 40, 40, 40, 300, 0), (7, 3, 1, 33, 64, 128),
    (130, 8, 8, 64, 96, None), (1, 1, 1, 1, 3, 2), (9, 12, 4, 128, 0, 500), (600, 2, 1, 16, 20, None), (1, 33, 1, 128, 700, 129)])
def test_sizes(S, H, KV, dim, cap, prefix, dtype):
    run(make(S, H, KV, dim, cap, prefix, dtype, seed=S + cap))


@TYPES
@pytest.mark.parametrize("cap,prefix", [(20000, None), (300, 20000), (0, 9000)])
def test_long(cap, prefix, dtype):
    run(make(3, 4, 2, 64, cap, prefix, dtype, seed=cap))


@TYPES
def test_nothing_to_attend_to(dtype):
    c = make(4, 4, 2, 64, 50, None, dtype, seed=1)
    c["lengths"][:] = torch.tensor([0, 3, 0, -7], dtype=torch.int32)
    run(c)
    c = make(2, 4, 2, 64, 0, None, dtype, seed=2)
    assert bool((run(c) == 0).all())
    c = make(0, 4, 2, 64, 10, 5, dtype, seed=3)
    assert ops.attention_step(**c).shape == (0, 4, 64)


@TYPES
@pytest.mark.parametrize("prefix", [None, 40])
def test_places_behind_the_length_reach_nothing(prefix, dtype):
    c = make(6, 4, 2, 100, 300, prefix, dtype, seed=4)
    clean = ops.attention_step(**c)
    for s in range(6):
        n = int(c["lengths"][s])
        c["k"][s, n:], c["v"][s, n:] = math.nan, math.inf
    assert torch.equal(run(c), clean)
    c["lengths"][2] = 400                                                     # the capacity: it was that already
    assert torch.equal(ops.attention_step(**c), clean)
    c["v"][3, 0] = math.nan                                                   # another sequence's own
    c["lengths"][3] = 200
    got = ops.attention_step(**c)
    assert torch.equal(got[[0, 1, 2, 4, 5]], clean[[0, 1, 2, 4, 5]]) and bool(got[3].isnan().all())


@TYPES
@pytest.mark.parametrize("scale", [0.0, 1.0, 25.0])
def test_scales(scale, dtype):
    run(make(4, 4, 2, 64, 400, 100, dtype, seed=5), scale=scale)


@TYPES
def test_parts_whose_scores_lie_far_apart(dtype):
    c = make(3, 2, 1, 32, 3000, 1000, dtype, seed=6)
    c["q"].fill_(1.0)
    c["k"].zero_()
    c["k"][:, :, 0, 0] = (torch.arange(3000, device=DEV) // 500 % 3).to(dtype) * 300 - 300
    c["prefix_k"].zero_()
    run(c, scale=1.0)


@TYPES
def test_strides(dtype):
    S, H, KV, dim, cap, P = 3, 4, 2, 40, 150, 70
    c = make(S, H, KV, dim, cap, P, dtype, seed=7)
    want = run(c)
    heads_first = {n: c[n].transpose(1, 2).contiguous().transpose(1, 2) for n in ("k", "v")}
    kv = torch.zeros(S, cap, 2 * KV, dim + 3, dtype=dtype, device=DEV)[:, :, :, 1:1 + dim]
    kv[:, :, :KV], kv[:, :, KV:] = c["k"], c["v"]
    out = torch.full((S, H, dim + 2), 5.0, dtype=dtype, device=DEV)
    for over in (heads_first, dict(k=kv[:, :, :KV], v=kv[:, :, KV:]), dict(prefix_k=c["prefix_k"].transpose(0, 1).contiguous().transpose(0, 1)),
                 dict(out=out[:, :, 1:-1])):
        assert torch.equal(ops.attention_step(**dict(c, **over)), want)
    assert bool((out[:, :, 0] == 5).all()) and bool((out[:, :, -1] == 5).all())
    same = dict(c, k=c["k"][:1].expand(S, cap, KV, dim), v=c["v"][:1].expand(S, cap, KV, dim))             # one cache for all
    run(same)


@TYPES
@pytest.mark.parametrize("group", [1, 4])
def test_the_last_row_of_a_prompt(group, dtype):
    """What a step gives is what attention gives for the same token at the end of its sequence."""
    KV, dim, P, n = 2, 64, 130, 45
    g = torch.Generator(device=DEV).manual_seed(8)
    t = lambda h: torch.randn(P + n, h, dim, device=DEV, generator=g).to(dtype)  # noqa: E731
    q, k, v = t(KV * group), t(KV), t(KV)
    off = torch.tensor([0, P + n], dtype=torch.int64, device=DEV)
    full = ops.attention(q, k, v, off).o[-1]
    lengths = torch.tensor([n], dtype=torch.int32, device=DEV)
    step = ops.attention_step(q[-1:], k[None, P:], v[None, P:], lengths, prefix_k=k[:P], prefix_v=v[:P])[0]
    # both are within r + u of the value's size of the same value, and sum other orders: 2 (r + dim u + n u) of sum p |v| <= max |v|
    r = 2.0 ** -8 if dtype == B16 else 0.0
    assert float((full.double() - step.double()).abs().max()) <= 2 * (2 * r + (dim + P + n + 100) * 4 * U) * float(v.abs().max())


@TYPES
def test_the_same_call_gives_the_same_bits(dtype):
    c = make(20, 8, 2, 128, 700, 900, dtype, seed=9)
    first = ops.attention_step(**c)
    for _ in range(5):
        assert torch.equal(ops.attention_step(**c), first)


def test_refusals():
    c = make(2, 4, 2, 16, 30, 10, F32, seed=10)
    wide = dict(q=torch.zeros(2, 4, 136, device=DEV), k=torch.zeros(2, 30, 2, 136, device=DEV), v=torch.zeros(2, 30, 2, 136, device=DEV), prefix_k=None,
                prefix_v=None)
    for over, word in [(dict(q=c["q"][0]), "indices"), (dict(k=c["k"][:1]), "shape"), (dict(v=c["v"].to(B16)), "float32"),
                       (dict(lengths=c["lengths"].long()), "int32"), (dict(lengths=c["lengths"][:1]), "shape"), (dict(prefix_k=None), "missing"),
                       (dict(prefix_v=c["prefix_v"][:5]), "shape"), (dict(q=c["q"][:, :3]), "multiple"), (wide, "dim"), (dict(scale=-1.0), "scale"),
                       (dict(scale=math.nan), "scale"), (dict(out=c["q"]), "lies over"), (dict(out=c["k"][:, 0]), "shape"),
                       (dict(q=c["q"].clone().requires_grad_()), "gradient")]:
        with pytest.raises(lsam.LsamError) as e:
            ops.attention_step(**dict(c, **over))
        assert e.value.code == lsam.EINVAL and word in str(e.value), (word, str(e.value))
