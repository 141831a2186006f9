"""lsam_residual without an eps, for rows whose mean square is no normal number of fp32: n(x) is 0 there as it is where squares pass the range, nothing is NaN,
and gradients of the weights keep what other rows give.  Just inside of the range values are those of the definition; the reference and the
tolerances are those of test_gpu_residual."""
import pytest
import torch

from paper_2509_03110_amd import ops

from test_gpu_residual import B16, DEV, F32, check, make  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [F32, B16])
DIMS = pytest.mark.parametrize("dim", [8, 70, 1024, 2000, 5000, 16384])


@TYPES
@DIMS
@pytest.mark.parametrize("small", [0.0, 1e-25, 1e-30, 1e-38])
def test_rows_that_vanish(small, dim, dtype):
    case, dr, dh = make(1, 9, dim, dtype, seed=dim)
    gone, rest = [0, 4], [1, 2, 3, 5, 6, 7, 8]
    kw = dict(w_post=case["w_post"], gate=case["gate"], eps=0.0)
    case["y"][:, gone] = small
    new, h = ops.residual(case["r"], case["y"], case["w_pre"], **kw)
    assert torch.equal(new[:, gone], case["r"][:, gone]) and bool(h.isfinite().all())
    new[:, gone] = small
    _, h = ops.residual(new, None, case["w_pre"], eps=0.0)
    assert bool((h[:, gone] == 0).all())
    got = ops.residual_backward(new, case["y"], case["w_pre"], dr, dh, **kw)
    assert all(bool(t.isfinite().all()) for t in got)
    # no norm there: the stream's gradient goes through, the others' is 0
    assert torch.equal(got.dr[:, gone], dr[:, gone]) and bool((got.dy[:, gone] == 0).all()) and bool((got.dgate[:, gone] == 0).all())
    # the others as without those rows
    few = ops.residual_backward(new[:, rest], case["y"][:, rest], case["w_pre"], dr[:, rest], dh[:, rest], w_post=case["w_post"],
                                gate=case["gate"][:, rest], eps=0.0)
    for n in ("dr", "dy", "dgate"):
        assert torch.equal(getattr(got, n)[:, rest], getattr(few, n)), n
    for n in ("dw_pre", "dw_post"):                                              # rows are added in their order: zeros in between change no rounding
        assert torch.equal(getattr(got, n), getattr(few, n)), n


@DIMS
@pytest.mark.parametrize("size", [2e-19, 1e-18, 1e16])
def test_rows_within_the_range(size, dim):
    """Squares from 2^-126 on: where a row's mean is a normal number all that underflow takes from its terms is below half a step of it."""
    case, dr, dh = make(1, 6, dim, F32, seed=dim + 1)
    case["y"][:, 2] = size * (1 + torch.rand(dim, device=DEV))
    case["r"].mul_(size)
    case["r"].copy_(case["r"] + size)
    for t in (dr, dh):
        t.mul_(1e-10)
    case["gate"] = None
    w_post, case["w_post"] = case["w_post"], None
    check(dict(case, y=None), dr, dh, eps=0.0)                                   # the norm of the stream
    case["w_post"] = w_post
    case["r"].zero_()
    check(case, dr, dh, eps=0.0)                                                 # that of y
