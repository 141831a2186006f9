"""The operators at sizes where a call becomes several launches, or a launch nears the most lanes that it can have.  Cases that need
more memory than is free are skipped."""
import pytest
import torch

from paper_2509_03110_amd import ops
from test_gpu_dropout import philox

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B16 = torch.bfloat16


@pytest.fixture(autouse=True)
def room():
    """Memory that other tests left in the allocator, and afterwards what these leave."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def need(gib):
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip("%d GiB of free memory are needed" % gib)


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


def test_short_segments_of_very_many_rows():
    # segments of 16 rows: tiles of 16 rows would be 2^23 workgroups of 512 lanes
    need(24)
    rows, inp, out, n = (1 << 27) + 40, 8, 8, (1 << 23) + 4
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randint(-4, 5, (rows, inp), device=DEV, generator=g, dtype=torch.int8).to(B16)      # whole numbers: sums are exact
    W = torch.randint(-4, 5, (out, inp), device=DEV, generator=g).to(B16)
    A, B = (torch.randint(-2, 3, s, device=DEV, generator=g).to(B16) for s in ((3, 1, inp), (3, out, 1)))
    sb = (torch.arange(n + 1, device=DEV, dtype=torch.int64) * 16).clamp(max=rows).int()
    which = (torch.arange(n, device=DEV) % 4 - 1).int()
    y, u = ops.adapter(x, W, A, B, sb, which, 1.0)
    for lo in (0, (1 << 26) - 100, (1 << 27) - 300, rows - 300):
        r = torch.arange(lo, lo + 300, device=DEV)
        a = which[r // 16].long()
        xs = x[lo:lo + 300].float()
        v = (xs[:, None, :] * A.float()[a.clamp(min=0), 0][:, None, :]).sum(2) * (a >= 0)[:, None]
        assert torch.equal(u[lo:lo + 300], v)
        want = (xs[:, None, :] * W.float()).sum(2) + v * B.float()[a.clamp(min=0), :, 0]
        assert torch.equal(y[lo:lo + 300], want.to(B16))


def test_copies_of_more_numbers_than_a_launch_has_lanes_for():
    # rows of 129 numbers are copied to rows of 136: 2^32 lanes of eight numbers at these rows
    need(160)
    rows, inp = 254_000_000, 129
    x = torch.zeros(rows, inp, device=DEV, dtype=B16)
    marked = torch.tensor([0, 5, 126_000_000, rows - 900_000, rows - 1], device=DEV)
    x[marked] = 1
    W = torch.ones(1, inp, device=DEV, dtype=B16)
    A, B = torch.ones(1, 1, inp, device=DEV, dtype=B16), torch.ones(1, 1, 1, device=DEV, dtype=B16)
    sb, which = torch.tensor([rows - 10, rows], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    y, u = ops.adapter(x, W, A, B, sb, which, 1.0)
    assert torch.equal(y[marked, 0].float(), torch.tensor([129.0, 129, 129, 129, 258], device=DEV).to(B16).float())
    assert int((y != 0).sum()) == 5 and int((u != 0).sum()) == 1


def test_log_probabilities_of_more_rows_than_a_launch_takes():
    rows, V = (1 << 23) + 37, 3
    g = torch.Generator(device=DEV).manual_seed(3)
    z = torch.randn(rows, V, device=DEV, generator=g)
    tokens = torch.randint(0, V, (rows,), device=DEV, generator=g, dtype=torch.int32)
    r = ops.logprobs(z, tokens, top=2)
    gl, ge = torch.randn(rows, device=DEV, generator=g), torch.randn(rows, device=DEV, generator=g)
    dz = ops.logprobs_backward(z, tokens, r.lse, r.entropy, gl, ge)
    for rows_of in (slice(0, 50), slice((1 << 23) - 50, rows)):
        part = ops.logprobs(z[rows_of], tokens[rows_of], top=2)
        for p, q in zip(r, part):
            assert torch.equal(p[rows_of], q)
        assert torch.equal(dz[rows_of], ops.logprobs_backward(z[rows_of], tokens[rows_of], part.lse, part.entropy, gl[rows_of], ge[rows_of]))


@pytest.mark.parametrize("length", [1, 2, 20])
def test_more_sequences_than_a_launch_takes(length):
    # workgroups of one wavefront: 2^22 - 8 sequences a launch; of eight: 2^19 - 8
    S = (1 << 22) + 11 if length < 20 else (1 << 19) + 11
    g = torch.Generator(device=DEV).manual_seed(4)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    f, x, dh = (n(S, length, 1) for _ in range(3))
    h0, dlast = n(S, 1), n(S, 1)
    r = ops.recurrence(f, x, h0=h0, save=True)
    got = (r.h, r.last) + ops.recurrence_backward(f, x, dh, r.states, h0=h0, dlast=dlast)
    for part in (slice(0, 300), slice(S - 300, S)):
        q = ops.recurrence(f[part], x[part], h0=h0[part], save=True)
        want = (q.h, q.last) + ops.recurrence_backward(f[part], x[part], dh[part], q.states, h0=h0[part], dlast=dlast[part])
        assert all(torch.equal(p[part], w) for p, w in zip(got, want))


def test_dropout_of_more_pieces_than_a_launch_takes():
    need(14)
    rows, step, site = (1 << 31) - 1, 4, 2                  # a launch takes 2^31 - 256 pieces, a row of one column each
    x = torch.ones(rows, 1, device=DEV, dtype=B16)
    y = ops.dropout(x, 0.5, 3, step, site=site)
    for lo in (0, (1 << 31) - 456, rows - 200):
        keep = [philox((0, r, site, step), (3, 0))[0] & 0xFFFF >= 1 << 15 for r in range(lo, lo + 200)]
        assert y[lo:lo + 200, 0].tolist() == [2.0 if k else 0.0 for k in keep]
