"""Operators whose arguments are parts of one array, side by side: what a fused projection gives, and what its gradient wants."""
import pytest
import torch

from paper_2509_03110_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(*shape, device=DEV, generator=g).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lead,offsets", [((3, 1), None), ((3, 40), None), ((1, 2000), None), ((500,), [0, 20, 300, 500])])
def test_gates_and_inputs_of_one_projection(dtype, lead, offsets):
    D = 33
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int64, device=DEV)
    fx, dh = rand(*lead, 2 * D, dtype=dtype, seed=1), rand(*lead, D, dtype=dtype, seed=2)
    f, x = fx[..., :D], fx[..., D:]
    r = ops.recurrence(f, x, offsets=off, save=True)
    df, dx, dh0 = ops.recurrence_backward(f, x, dh, r.states, offsets=off)
    both = torch.empty_like(fx)
    df2, dx2, _ = ops.recurrence_backward(f, x, dh, r.states, offsets=off, df=both[..., :D], dx=both[..., D:])
    assert torch.equal(both, torch.cat((df, dx), -1)) and torch.equal(df2, df) and torch.equal(dx2, dx)
    wide = torch.zeros(*lead, 3 * D, device=DEV, dtype=dtype)
    wide[..., :D], wide[..., D:2 * D] = f, x
    q = ops.recurrence(wide[..., :D], wide[..., D:2 * D], offsets=off, out=wide[..., 2 * D:])
    assert torch.equal(q.h, r.h) and torch.equal(wide[..., :2 * D], fx)


@pytest.mark.parametrize("rows", [7, 100])
def test_results_beside_their_inputs(rows):
    inp, out = 40, 24
    xy = rand(rows, inp + out, dtype=torch.bfloat16, seed=3)
    W, A, B = rand(out, inp, dtype=torch.bfloat16, seed=4), rand(2, 4, inp, dtype=torch.bfloat16, seed=5), rand(2, out, 4, dtype=torch.bfloat16, seed=6)
    sb = torch.tensor([0, 3, rows], dtype=torch.int32, device=DEV)
    sa = torch.tensor([1, 0], dtype=torch.int32, device=DEV)
    want, _ = ops.adapter(xy[:, :inp].contiguous(), W, A, B, sb, sa, 1.0)
    ops.adapter(xy[:, :inp], W, A, B, sb, sa, 1.0, out=xy[:, inp:])
    assert torch.equal(xy[:, inp:], want)
    t = rand(2, rows, 2 * inp, dtype=torch.float32, seed=7)
    want = ops.dropout(t[:, :, :inp].contiguous(), 0.5, 1, 2)
    ops.dropout(t[:, :, :inp], 0.5, 1, 2, out=t[:, :, inp:])
    assert torch.equal(t[:, :, inp:], want)
