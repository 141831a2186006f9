"""The gradient of lsam_residual where a workgroup walks over several rows (there are some 1024 workgroups for all replicas), for every number of
wavefronts that a row takes.  The reference and the tolerances are those of test_gpu_residual."""
import pytest
import torch

from paper_2509_03110_amd import ops

from test_gpu_residual import B16, F32, check, make  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [F32, B16])


@TYPES
@pytest.mark.parametrize("K,rows,dim", [(1, 2060, 512), (1, 1025, 1000), (1, 3100, 1025), (2, 1100, 2048), (1, 1100, 4096), (3, 1033, 4001), (1, 1100, 8192), (40, 80, 5003),
                                        (1, 1100, 16384), (1, 1026, 9001), (16, 200, 8193), (700, 7, 2050)])
def test_rows_of_a_workgroup(K, rows, dim, dtype):
    case, dr, dh = make(K, rows, dim, dtype, seed=rows + dim)
    check(case, dr, dh)


@TYPES
@pytest.mark.parametrize("left_out", [("gate",), ("w_post",), ("gate", "w_post"), ("w_pre",), ("y",), ("w_pre", "gate", "w_post"), ("dr",), ("dr", "y")])
@pytest.mark.parametrize("dim", [900, 3001, 9001])
def test_parts_that_are_not_there(dtype, left_out, dim):
    case, dr, dh = make(1, 2100, dim, dtype, seed=len(left_out) + dim, gate="gate" not in left_out, y="y" not in left_out)
    for name in left_out:
        if name in case:
            case[name] = None
    check(case, None if "dr" in left_out else dr, dh)


@TYPES
@pytest.mark.parametrize("dim", [100, 4096, 16384])
def test_each_row_as_by_itself(dim, dtype):
    """Rows of a long call have the bits that they have in a call of few, where a workgroup has one; and dr_out over dr changes none."""
    case, dr, dh = make(1, 2050, dim, dtype, seed=dim)
    kw = dict(w_post=case["w_post"], gate=case["gate"], alpha=0.75, beta=-0.5)
    all_rows = ops.residual_backward(case["r"], case["y"], case["w_pre"], dr, dh, **kw)
    for lo, hi in ((0, 7), (1020, 1030), (2043, 2050)):
        cut = slice(lo, hi)
        few = ops.residual_backward(case["r"][:, cut], case["y"][:, cut], case["w_pre"], dr[:, cut], dh[:, cut], **dict(kw, gate=case["gate"][:, cut]))
        assert all(torch.equal(getattr(few, n), getattr(all_rows, n)[:, cut]) for n in ("dr", "dy", "dgate"))
    again = dr.clone()
    over = ops.residual_backward(case["r"], case["y"], case["w_pre"], again, dh, dr_out=again, **kw)
    assert all(torch.equal(a, b) for a, b in zip(over, all_rows))
