"""lsam_dropout against a plain computation in 64 bits.

The mask is a whole-number computation and has to be equal.  A kept value is one product and one sum in fp32,
rounded once: at most 2 units of 2^-24 of |x scale| + |residual| in fp32, and the rounding of eight significant bits (2^-8) more
where the result is stored as bfloat16."""
import numpy as np
import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def philox(c, k):
    """Philox4x32-10 on Python integers."""
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(K, rows, cols, p, seed, step, site, first):
    drop = round(p * 65536)
    m = np.zeros((K, rows, cols), bool)
    for k in range(K):
        for r in range(rows):
            for g in range((cols + 7) // 8):
                w = philox((g, r, site | (first + k) << 16, step), (seed & 0xFFFFFFFF, seed >> 32))
                for e in range(min(8, cols - 8 * g)):
                    m[k, r, 8 * g + e] = (w[e // 2] >> 16 * (e % 2)) & 0xFFFF >= drop
    return m


def check(y, x, res, m, p):
    scale = 65536 / (65536 - round(p * 65536)) if round(p * 65536) < 65536 else 0.0
    kept_x = np.where(m, x.double().cpu().numpy(), 0.0) * scale
    r = 0.0 if res is None else res.double().cpu().numpy()
    unit = 2.0 ** -24 * 2 + (2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0)
    got = y.double().cpu().numpy()
    assert np.all(np.abs(got - (kept_x + r)) <= unit * (np.abs(kept_x) + np.abs(r)) + 1e-38)
    if res is None:
        assert np.all(got[~m] == 0.0)


def test_the_generator_gives_the_published_numbers():
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K,rows,cols,pad,p,res,shift", [
    (1, 1, 1, 0, 0.5, False, 0), (2, 3, 8, 0, 0.1, True, 0), (3, 5, 17, 3, 0.25, True, 1), (1, 40, 129, 1, 0.5, False, 1),
    (2, 2, 784, 0, 0.9, False, 0), (1, 7, 64, 0, 0.0, True, 0), (2, 4, 9, 0, 1.0, True, 0), (1, 1, 4099, 5, 1e-4, False, 1)])
def test_dropout_matches_the_definition(dtype, K, rows, cols, pad, p, res, shift):
    g = torch.Generator(device=DEV).manual_seed(K * 1000 + cols)
    seed, step, site, first = 0x123456789ABCDEF0 + cols, 70000 + rows, 5, 2

    def make():
        flat = torch.randn(K * rows * (cols + pad) + shift, device=DEV, generator=g).to(dtype)
        return flat[shift:].view(K, rows, cols + pad)[:, :, :cols]
    x, r = make(), make() if res else None
    keep = x.clone()
    y = ops.dropout(x, p, seed, step, site=site, first_replica=first, residual=r)
    m = kept(K, rows, cols, p, seed, step, site, first)
    check(y, x, r, m, p)
    assert torch.equal(x, keep)
    # in place, into a strided array whose padding stays as it was, and replica by replica
    base = torch.full((K, rows, cols + 3), 7.0, device=DEV, dtype=dtype)
    out = base[:, :, :cols]
    out.copy_(x)
    ops.dropout(out, p, seed, step, site=site, first_replica=first, residual=r, out=out)
    assert torch.equal(out, y) and bool((base[:, :, cols:] == 7.0).all())
    for k in range(K):
        yk = ops.dropout(x[k], p, seed, step, site=site, first_replica=first + k, residual=None if r is None else r[k])
        assert torch.equal(yk, y[k])


def test_the_mask_depends_on_each_of_its_coordinates_and_has_the_rate_asked_for():
    x = torch.ones(4, 512, 512, device=DEV)
    a = ops.dropout(x, 0.3, 1, 1)
    rate = float((a == 0).double().mean())
    assert abs(rate - 0.3) < 5 * (0.3 * 0.7 / x.numel()) ** 0.5 + 1 / 65536
    for other in (dict(seed=2, step=1), dict(seed=1 + (1 << 32), step=1), dict(seed=1, step=2), dict(seed=1, step=1, site=1),
                  dict(seed=1, step=1, first_replica=4)):
        b = ops.dropout(x, 0.3, **other)
        both = float(((a == 0) & (b == 0)).double().mean())
        assert abs(both - 0.09) < 5 * (0.09 * 0.91 / x.numel()) ** 0.5 + 1 / 65536
    assert torch.equal(a, ops.dropout(x, 0.3, 1, 1))


def test_dropped_values_are_zero_whatever_they_were_and_kept_ones_stay():
    x = torch.full((1, 64, 64), float("nan"), device=DEV)
    x[0, ::2] = float("inf")
    y = ops.dropout(x, 0.5, 3, 4)
    m = torch.from_numpy(kept(1, 64, 64, 0.5, 3, 4, 0, 0)).to(DEV)
    assert bool((y[~m] == 0).all()) and bool(y[0, 1::2][m[0, 1::2]].isnan().all()) and bool(y[0, ::2][m[0, ::2]].isinf().all())
    assert bool((ops.dropout(x, 1.0, 3, 4) == 0).all())


def test_the_gradient_is_the_same_mask_and_agrees_with_differences():
    x = torch.randn(2, 9, 33, device=DEV, dtype=torch.float32)
    dy, e = torch.randn_like(x), torch.randn_like(x)
    dx = ops.dropout(dy, 0.25, 11, 12, site=3)
    f = lambda t: float((ops.dropout(t, 0.25, 11, 12, site=3).double() * dy.double()).sum())  # noqa: E731
    # linear in x: the difference quotient is exact up to the rounding of 594 fp32 products and sums
    terms = float((ops.dropout(e, 0.25, 11, 12, site=3).double() * dy.double()).abs().sum())
    diff = f(x + e) - f(x)
    size = float((ops.dropout(x, 0.25, 11, 12, site=3).double() * dy.double()).abs().sum()) + terms
    assert abs(diff - float((dx.double() * e.double()).sum())) <= 4 * 2.0 ** -24 * (2 * size + terms)


def test_a_call_runs_on_the_stream_it_is_given_and_in_a_graph():
    x = torch.randn(4, 100, 200, device=DEV)
    want = ops.dropout(x, 0.5, 1, 2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ops.dropout(x, 0.5, 1, 2, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.dropout(x, 0.5, 1, 2, out=out)
    for n in range(3):
        x.copy_(torch.randn(4, 100, 200, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ops.dropout(x, 0.5, 1, 2))


def test_refusals():
    x = torch.zeros(2, 4, 16, device=DEV)
    for bad in (dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(seed=1 << 64), dict(step=1 << 32), dict(site=1 << 16),
                dict(first_replica=65535), dict(residual=x[:, :, :8]), dict(residual=x.double()), dict(out=x.bfloat16()),
                dict(residual=x.cpu()), dict(x=x.half()), dict(x=x.cpu()), dict(x=x.transpose(1, 2)), dict(x=x[None])):
        kw = dict(dict(x=x, p=0.5, seed=1, step=1), **bad)
        with pytest.raises(lsam.LsamError) as e:
            ops.dropout(**kw)
        assert e.value.code == lsam.EINVAL
    flat = torch.zeros(200, device=DEV)
    with pytest.raises(lsam.LsamError) as e:
        ops.dropout(flat[:64].view(1, 4, 16), 0.5, 1, 1, out=flat[8:72].view(1, 4, 16))
    assert "lies over" in str(e.value)
    assert ops.dropout(torch.zeros(2, 0, 16, device=DEV), 0.5, 1, 1).shape == (2, 0, 16)
