"""The operators at sizes where a call becomes several launches, or a launch nears the most lanes that it can have."""
import pytest
import torch

from paper_2509_03110_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B16 = torch.bfloat16


@pytest.fixture(autouse=True)
def room():
    """Memory that other tests left in the allocator, and afterwards what these leave."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_more_adapters_times_outputs_than_a_launch_has_lanes():
    # 65535 x 65552 > 2^32; all adapters but two are the same memory
    rows, inp, out, m = 65, 8, 65552, 65535
    g = torch.Generator(device=DEV).manual_seed(1)
    x, W = torch.randn(rows, inp, device=DEV, generator=g).to(B16), torch.randn(out, inp, device=DEV, generator=g).to(B16)
    A, B = torch.randn(1, 2, inp, device=DEV, generator=g).to(B16), torch.randn(1, out, 2, device=DEV, generator=g).to(B16)
    sb = torch.tensor([0, 30, 65], dtype=torch.int32, device=DEV)
    which = torch.tensor([m - 1, 7], dtype=torch.int32, device=DEV)
    y, u = ops.adapter(x, W, A.expand(m, 2, inp), B.expand(m, out, 2), sb, which, 0.5)
    want, wu = ops.adapter(x, W, A, B, sb, torch.zeros_like(which), 0.5)
    assert torch.equal(u, wu) and torch.equal(y, want)
    dy = torch.randn(rows, out, device=DEV, generator=g).to(B16)
    dx = ops.adapter_backward(x, W, A.expand(m, 2, inp), B.expand(m, out, 2), u, dy, sb, which, 0.5, want_adapters=False)[0]
    assert torch.equal(dx, ops.adapter_backward(x, W, A, B, u, dy, sb, torch.zeros_like(which), 0.5, want_adapters=False)[0])
