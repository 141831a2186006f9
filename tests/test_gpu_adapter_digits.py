"""lsam_adapter with bf16 rows: what is held in fp32 -- u, du, and adapters where they are -- keeps all of its digits.

Every number here is a sum of three powers of two at most 2^21 apart, and so is every sum of products on the way, in any order: fp32
holds them all, and the result, a power of two, is a bfloat16.  So results are equal to the definition's, not near them: the
leading digits of the low-rank term cancel against x W^T, and what is left is what its last digits make."""
import pytest
import torch

from paper_2509_03110_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, B16 = torch.float32, torch.bfloat16
M, L = 2.0 ** -9, 2.0 ** -20                       # digits of the second and the third bfloat16 piece of 1 + M + L


def segs(rows):
    return (torch.tensor([0, rows // 2, rows], dtype=torch.int32, device=DEV), torch.tensor([0, 1], dtype=torch.int32, device=DEV))


def zeros(*shape, t):
    return torch.zeros(*shape, device=DEV, dtype=t)


SIZES = [(5, 8, 40), (64, 40, 40), (40, 8, 8400), (65, 8, 40), (300, 24, 72), (4000, 8, 3900)]


@pytest.mark.parametrize("atype", [F32, B16])
@pytest.mark.parametrize("rows,inp,out", SIZES)
def test_last_digits_of_u_reach_the_result(rows, inp, out, atype):
    x, W, A, B = zeros(rows, inp, t=B16), zeros(out, inp, t=B16), zeros(2, 5, inp, t=atype), zeros(2, out, 5, t=atype)
    x[:, :3] = 1
    A[:, 2, 0], A[:, 2, 1], A[:, 2, 2] = 1, M, L     # u = 1 + M + L
    B[:, :, 2] = 1
    W[:, 0], W[:, 1] = -1, -M
    y, u = ops.adapter(x, W, A, B, *segs(rows), 1.0)
    assert bool((u[:, 2] == 1 + M + L).all()) and bool((y == L).all())


@pytest.mark.parametrize("rows,inp,out", SIZES)
def test_last_digits_of_fp32_adapters_reach_the_result(rows, inp, out):
    x, W, A, B = zeros(rows, inp, t=B16), zeros(out, inp, t=B16), zeros(2, 5, inp, t=F32), zeros(2, out, 5, t=F32)
    x[:, :3] = 1
    A[:, 1, 0] = 1
    B[:, :, 1] = 1 + M + L
    W[:, 0], W[:, 1] = -1, -M
    y, _ = ops.adapter(x, W, A, B, *segs(rows), 1.0)
    assert bool((y == L).all())
    A[:, 1, 0], B[:, :, 1] = 1 + M, 1 + M            # 1 + 2 M + M^2: the product of both second pieces
    W[:, 0], W[:, 1] = -1, -2 * M
    y, _ = ops.adapter(x, W, A, B, *segs(rows), 1.0)
    assert bool((y == M * M).all())


@pytest.mark.parametrize("atype", [F32, B16])
@pytest.mark.parametrize("rows,out,inp", SIZES)
def test_last_digits_of_du_and_A_reach_the_gradient(rows, out, inp, atype):
    x, W, A, B = zeros(rows, inp, t=B16), zeros(out, inp, t=B16), zeros(2, 5, inp, t=atype), zeros(2, out, 5, t=atype)
    u, dy = zeros(rows, 5, t=F32), zeros(rows, out, t=B16)
    dy[:, :3] = 1
    B[:, 0, 2], B[:, 1, 2], B[:, 2, 2] = 1, M, L     # du = 1 + M + L
    A[:, 2, :] = 1
    W[0, :], W[1, :] = -1, -M
    dx, _, _ = ops.adapter_backward(x, W, A, B, u, dy, *segs(rows), 1.0, want_adapters=False)
    assert bool((dx == L).all())
    if atype == F32:
        B[:, 1:, 2] = 0
        A[:, 2, :] = 1 + M + L
        dx, _, _ = ops.adapter_backward(x, W, A, B, u, dy, *segs(rows), 1.0, want_adapters=False)
        assert bool((dx == L).all())
