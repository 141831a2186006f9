"""lsam_residual and its gradient against the definition in 64 bits.

Tolerances (u = 2^-24): a sum over a row is at most 16 additions in a lane, 6 over the lanes and 15 over wavefronts, of products: 40 u of
the sum of absolute values.  1 / sqrt(mean + eps) halves that of its argument, and adds a division, a sum, a square root and a division:
25 u of itself; n(x) 26 u.  sigmoid and its complement are off by (1.5 |x| + 7) u of themselves (one power, a sum, a reciprocal, a product).  Every product
and sum beside these adds u of its result; sums of absolute values stand in for results that cancel.  Sums over rows: a group of workgroups adds
at most rows numbers one after the other: (rows + 40) u of the absolute values.  Stored in bfloat16: 2^-8 of itself.  h is held to the norm
of r' as it was stored."""
import math

import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, B16 = torch.float32, torch.bfloat16


def near(got, want, bound, what):
    bound = bound + (2.0 ** -8 * (want.abs() + bound) if got.dtype == B16 else U * want.abs()) + 1e-37
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (what, float((off / bound).max()))


def reference(r, y, w_pre, w_post, gate, alpha, beta, eps, new=None, dr=None, dh=None):
    """{name: (value, bound)}; with `new` (r' as stored) what depends on it."""
    wide = lambda t: None if t is None else t.double()  # noqa: E731
    r, y, gate, new, dr, dh = (wide(t) for t in (r, y, gate, new, dr, dh))
    K, rows, dim = r.shape
    each = lambda w: None if w is None else wide(w).reshape(-1, 1, dim)  # noqa: E731
    w_pre, w_post = each(w_pre), each(w_post)
    mean = lambda t: t.mean(2, keepdim=True)  # noqa: E731
    inv = lambda t: 1 / torch.sqrt(mean(t * t) + eps)  # noqa: E731
    out = {}
    one = torch.ones((), dtype=torch.float64, device=DEV)
    s, rest, es = one, 0 * one, 0 * one
    if gate is not None:
        s, rest = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
        es = (1.5 * gate.abs() + 7) * U
    n = iy = v = None
    if y is not None:
        iy = inv(y) if w_post is not None else one
        n, v = y * iy, w_post if w_post is not None else one
        o = n * v * s
        out["r"] = (alpha * r + beta * o, U * (2 * (alpha * r).abs() + (beta * o).abs() * 32) + es * (beta * o).abs())
    if new is None:
        return out
    if w_pre is not None:
        out["h"] = (new * inv(new) * w_pre, 28 * U * (new * inv(new) * w_pre).abs())
    if dh is None and dr is None:
        return out
    d = dr if dr is not None else 0 * new
    ed = U * d.abs()
    if w_pre is not None:
        i, m, g = inv(new), new * inv(new), dh * w_pre
        dot, size = mean(g * m), mean((g * m).abs())
        d = d + i * (g - m * dot)
        ed = ed + U * d.abs() + i * U * (30 * g.abs() + (60 + 30) * m.abs() * size + 30 * (m * dot).abs())
        out["dw_pre"] = ((dh * m).sum(1), ((rows + 70) * U * (dh * m).abs()).sum(1))
    a = alpha if y is not None else 1.0
    out["dr"] = (a * d, abs(a) * ed + U * (a * d).abs())
    if y is not None:
        part, ep = beta * d * s, abs(beta) * s * ed + (beta * d * s).abs() * (es + 3 * U)
        out["dgate"] = (beta * d * n * v * s * rest, abs(beta) * (n * v).abs() * s * rest * ed + (beta * d * n * v * s * rest).abs() * (2 * es + 34 * U))
        out["dw_post"] = ((part * n).sum(1), (ep * n.abs() + (part * n).abs() * (rows + 70) * U).sum(1))
        g, eg = part * v, ep * v.abs() + U * (part * v).abs()
        if w_post is not None:
            dot, size, more = mean(g * n), mean((g * n).abs()), mean(eg * n.abs())
            out["dy"] = (iy * (g - n * dot), iy * (eg + n.abs() * more + U * (30 * g.abs() + 90 * n.abs() * size + 30 * (n * dot).abs())))
        else:
            out["dy"] = (g, eg)
    return out


def make(K, rows, dim, dtype, seed, gate=True, y=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    x = lambda: n(K, rows, dim).to(dtype)  # noqa: E731
    return dict(r=(n(K, rows, dim) * 3).to(dtype), y=x() if y else None, gate=(2 * x()) if gate and y else None,
                w_pre=1 + 0.3 * n(K, dim), w_post=1 + 0.3 * n(K, dim)), x(), x()


def check(case, dr, dh, alpha=0.75, beta=-0.5, eps=1e-5):
    kw = dict(w_post=case["w_post"], gate=case["gate"], alpha=alpha, beta=beta, eps=eps)
    new, h = ops.residual(case["r"], case["y"], case["w_pre"], **kw)
    want = reference(**case, alpha=alpha, beta=beta, eps=eps, new=new, dr=dr, dh=dh)
    if case["y"] is not None:
        near(new, *want["r"], "r'")
    else:
        assert new is case["r"]
    if h is not None:
        near(h, *want["h"], "h")
    got = ops.residual_backward(new, case["y"], case["w_pre"], dr, dh if case["w_pre"] is not None else None, **kw)
    for name in ("dr", "dy", "dgate", "dw_pre", "dw_post"):
        t = getattr(got, name)
        lacks = dict(dr=False, dy=case["y"] is None, dgate=case["gate"] is None or case["y"] is None, dw_pre=case["w_pre"] is None,
                     dw_post=case["w_post"] is None or case["y"] is None)[name]
        assert (t is None) == lacks, name
        if t is not None:
            near(t, want[name][0].reshape(t.shape), want[name][1].expand_as(want[name][0]).reshape(t.shape), name)
    return new, h, got


SIZES = [(1, 1, 1), (2, 3, 7), (1, 5, 8), (3, 4, 513), (1, 9, 1000), (2, 2, 1024), (1, 3, 1025), (1, 2, 2049), (2, 3, 4096), (1, 2, 4100),
         (1, 2, 8192), (1, 2, 8200), (1, 1, 16384), (1, 1500, 40), (300, 2, 16)]


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("K,rows,dim", SIZES)
def test_all_parts(K, rows, dim, dtype):
    case, dr, dh = make(K, rows, dim, dtype, seed=rows + dim)
    check(case, dr, dh)


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("left_out", [("gate",), ("w_post",), ("gate", "w_post"), ("w_pre",), ("y",), ("w_pre", "gate", "w_post"), ("dr",),
                                      ("dr", "y")])
@pytest.mark.parametrize("dim", [24, 1100])
def test_parts_that_are_not_there(dtype, left_out, dim):
    case, dr, dh = make(2, 5, dim, dtype, seed=len(left_out) + dim, gate="gate" not in left_out, y="y" not in left_out)
    for name in left_out:
        if name in case:
            case[name] = None
    check(case, None if "dr" in left_out else dr, dh)


def test_gradients_against_differences():
    """The formula's own check: 64-bit differences of sum dr r' + dh h, by the reference alone, and the kernel against the formula above."""
    case, dr, dh = make(1, 2, 6, F32, seed=3)
    kw = dict(alpha=0.75, beta=-0.5, eps=1e-5)
    wide = {k: v.double() for k, v in case.items()}

    def value(c):
        new = reference(**c, **kw)["r"][0]
        return ((new * dr.double()) + reference(**c, **kw, new=new)["h"][0] * dh.double()).sum()
    new = reference(**wide, **kw)["r"][0]
    want = reference(**wide, **kw, new=new, dr=dr.double(), dh=dh.double())
    for name, key in (("r", "dr"), ("y", "dy"), ("gate", "dgate"), ("w_pre", "dw_pre"), ("w_post", "dw_post")):
        grad = want[key][0].reshape(wide[name].shape)
        for i in range(wide[name].numel()):
            step = torch.zeros_like(wide[name]).view(-1)
            step[i] = 1e-5
            up, down = (value({**wide, name: wide[name] + s * step.view_as(wide[name])}) for s in (1, -1))
            assert abs(float((up - down) / 2e-5 - grad.view(-1)[i])) < 1e-7 * (1 + abs(float(grad.view(-1)[i])))


@pytest.mark.parametrize("dtype", [F32, B16])
def test_strides_replicas_without_index_and_shared_weights(dtype):
    K, rows, dim, pad = 2, 6, 50, 3
    g = torch.Generator(device=DEV).manual_seed(8)
    wide = lambda: torch.randn(K, rows, dim + 2 * pad, device=DEV, generator=g).to(dtype)[:, :, pad:pad + dim]  # noqa: E731
    params = torch.randn(K, 500, device=DEV, generator=g)
    case = dict(r=wide(), y=wide(), gate=wide(), w_pre=params[:, 7:7 + dim], w_post=params[:, 111:111 + dim])
    dr, dh = wide(), wide()
    check(case, dr, dh)
    kw = dict(w_post=case["w_post"], gate=case["gate"])
    new, h = ops.residual(case["r"], case["y"], case["w_pre"], **kw)
    outs = [torch.full((K, rows, dim + 2 * pad), 5.0, device=DEV, dtype=dtype) for _ in range(2)]
    ops.residual(case["r"], case["y"], case["w_pre"], out=outs[0][:, :, pad:-pad], h=outs[1][:, :, pad:-pad], **kw)
    for t, want in zip(outs, (new, h)):
        assert torch.equal(t[:, :, pad:-pad], want) and bool((t[:, :, :pad] == 5).all()) and bool((t[:, :, -pad:] == 5).all())
    grads = torch.full((K, 500), 9.0, device=DEV)
    got = ops.residual_backward(new, case["y"], case["w_pre"], dr, dh, dw_pre=grads[:, 7:7 + dim], dw_post=grads[:, 111:111 + dim], **kw)
    again = ops.residual_backward(new, case["y"], case["w_pre"], dr, dh, **kw)
    assert torch.equal(grads[:, 7:7 + dim], again.dw_pre) and torch.equal(grads[:, 111:111 + dim], again.dw_post)
    assert bool((grads[:, :7] == 9).all()) and bool((grads[:, 7 + dim:111] == 9).all()) and bool((grads[:, 111 + dim:] == 9).all())
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # one replica, and weights that both share
    one = ops.residual(case["r"][1], case["y"][1], case["w_pre"][1], w_post=case["w_post"][1], gate=case["gate"][1])
    assert torch.equal(one[0], new[1]) and torch.equal(one[1], h[1])
    both = ops.residual(case["r"], case["y"], case["w_pre"][1], w_post=case["w_post"][1], gate=case["gate"])
    assert torch.equal(both[1][1], h[1])
    single = ops.residual_backward(new[1], case["y"][1], case["w_pre"][1], dr[1], dh[1], w_post=case["w_post"][1], gate=case["gate"][1])
    assert all(torch.equal(a, b[1]) for a, b in zip((single.dr, single.dy, single.dgate), (again.dr, again.dy, again.dgate)))


def test_in_place():
    case, dr, dh = make(2, 40, 300, B16, seed=4)
    kw = dict(w_post=case["w_post"], gate=case["gate"], alpha=0.5)
    new, h = ops.residual(case["r"], case["y"], case["w_pre"], **kw)
    r = case["r"].clone()
    got = ops.residual(r, case["y"], case["w_pre"], out=r, **kw)
    assert got[0] is r and torch.equal(r, new) and torch.equal(got[1], h)
    want = ops.residual_backward(new, case["y"], case["w_pre"], dr, dh, **kw)
    d = dr.clone()
    back = ops.residual_backward(new, case["y"], case["w_pre"], d, dh, dr_out=d, **kw)
    assert all(torch.equal(a, b) for a, b in zip(back, want)) and torch.equal(d, want.dr)


def test_what_is_not_finite_stays_in_its_row():
    case, dr, dh = make(1, 6, 70, F32, seed=5)
    clean = ops.residual(case["r"], case["y"], case["w_pre"], w_post=case["w_post"], gate=case["gate"])
    case["y"][0, 2, 3], case["r"][0, 4, 0], case["gate"][0, 5, 1] = math.nan, math.inf, -math.inf
    new, h = ops.residual(case["r"], case["y"], case["w_pre"], w_post=case["w_post"], gate=case["gate"])
    for row in (0, 1, 3):
        assert torch.equal(new[0, row], clean[0][0, row]) and torch.equal(h[0, row], clean[1][0, row])
    assert bool(new[0, 5].isfinite().all()) and bool(h[0, 2].isnan().all())
    got = ops.residual_backward(clean[0], case["y"], case["w_pre"], dr, dh, w_post=case["w_post"])
    assert bool(got.dy[0, [0, 1, 3, 4, 5]].isfinite().all()) and bool(got.dr.isfinite().all())


def test_a_row_of_zeros():
    r = torch.zeros(2, 9, device=DEV)
    w = torch.ones(9, device=DEV)
    new, h = ops.residual(r, r.clone(), w, w_post=w)
    assert bool((new == 0).all()) and bool((h == 0).all())
    got = ops.residual_backward(new, r, w, None, torch.ones_like(r), w_post=w)
    assert all(bool(t.isfinite().all()) for t in got if t is not None)


def test_no_rows():
    r, w = torch.empty(3, 0, 8, device=DEV), torch.ones(3, 8, device=DEV)
    new, h = ops.residual(r, r, w, w_post=w)
    assert new.shape == h.shape == r.shape
    got = ops.residual_backward(r, r, w, r, r, w_post=w)
    assert torch.equal(got.dw_pre, torch.zeros(3, 8, device=DEV)) and torch.equal(got.dw_post, torch.zeros(3, 8, device=DEV))


def test_refusals():
    case, dr, dh = make(2, 4, 16, F32, seed=6)
    r, y, w = case["r"], case["y"], case["w_pre"]
    for call, word in [(lambda: ops.residual(r[0, 0], None, w), "indices"), (lambda: ops.residual(r, y[:, :2], w), "shape"),
                       (lambda: ops.residual(r, y.to(B16), w), "float32"), (lambda: ops.residual(r, y, w[:1]), "shape"),
                       (lambda: ops.residual(r, y, w.to(B16)), "float32"), (lambda: ops.residual(r, None, None), "nothing to do"),
                       (lambda: ops.residual(r, y, w, eps=-1.0), "eps"), (lambda: ops.residual(r, y, w, eps=math.nan), "eps"),
                       (lambda: ops.residual(r, y, w, out=y), "lies over"), (lambda: ops.residual(r, y, w, h=r), "lies over"),
                       (lambda: ops.residual(r, y, w, out=r, h=r), "lies over"),
                       (lambda: ops.residual_backward(r, y, w, dr, None), "dh is missing"),
                       (lambda: ops.residual_backward(r, y, w[0], dr, dh), "shared"),
                       (lambda: ops.residual_backward(r, y, w, dr, dh, dr_out=dh), "lies over"),
                       (lambda: ops.residual_backward(r, y, w, dr, dh, dw_pre=w), "lies over"),
                       (lambda: ops.residual(torch.zeros(2, 16392, device=DEV), None, torch.zeros(16392, device=DEV)), "dim"),
                       (lambda: ops.residual(r, y.requires_grad_(), w), "gradient")]:
        with pytest.raises(lsam.LsamError) as e:
            call()
        assert e.value.code == lsam.EINVAL and word in str(e.value), (word, str(e.value))
