"""lsam_attention and its gradient where a wavefront's lanes hold the offsets of 60 sequences and more, and the last tile of rows is not whole: nothing is
written behind the last row, and values are those of the definition.  The reference and the tolerances are those of test_gpu_attention."""
import pytest
import torch

from paper_2509_03110_amd import ops

from test_gpu_attention import DEV, TYPES, check, make  # noqa: E402

pytestmark = pytest.mark.gpu
ROWS = 1000


def spread(n, rows=ROWS):
    return [rows * i // n for i in range(n + 1)]


OFFSETS = {"61": spread(61), "62": spread(62), "63": spread(63), "64": spread(64), "65": spread(65), "10 of 128": spread(10) + [ROWS] * 118,
           "3 of 66": spread(3) + [ROWS] * 63, "1 of 63": [0] + [ROWS] * 63, "rows behind": spread(63, 990), "all empty": [ROWS] * 64,
           "empty ones around": [0] * 40 + spread(5) + [ROWS] * 59}
# rows and heads shared by wavefronts and workgroups; each wavefront with rows, or keys, of its own; that with the heads of a group shared
HEADS = pytest.mark.parametrize("H,KV", [(4, 2), (52, 52), (80, 40)])


@TYPES
@pytest.mark.parametrize("offsets", OFFSETS.values(), ids=OFFSETS.keys())
@HEADS
def test_nothing_behind_the_last_row(H, KV, offsets, dtype):
    dim, behind = 32, 140
    q, k, v, do = make(ROWS, H, KV, dim, dtype, seed=len(offsets))
    want = check(q, k, v, do, offsets)
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    inside = slice(offsets[0], offsets[-1])

    def compare(whole, part):
        outs = [whole(h) for h in (H, H, KV, KV)]
        o, dq, dk, dv = (part(t) for t in outs)
        lse = ops.attention(q, k, v, off, save=True, out=o).lse
        ops.attention_backward(q, k, v, off, o, lse, do, dq=dq, dk=dk, dv=dv)
        assert torch.equal(lse[:, inside], want["lse"][:, inside])
        for t, of, n in zip(outs, (o, dq, dk, dv), ("o", "dq", "dk", "dv")):
            assert torch.equal(of[inside], want[n][inside]), n
            of[inside] = 7.0
            assert bool((t == 7).all()), n
    # rows behind the last; the next head's rows behind a head's last
    compare(lambda h: torch.full((ROWS + behind, h, dim), 7.0, dtype=dtype, device=DEV), lambda t: t[:ROWS])
    compare(lambda h: torch.full((h + 1, ROWS, dim), 7.0, dtype=dtype, device=DEV), lambda t: t[:-1].transpose(0, 1))


@TYPES
@pytest.mark.parametrize("rows,n", [(1, 63), (31, 63), (97, 63), (127, 64), (129, 63), (250, 63)])
@HEADS
def test_other_numbers_of_rows(H, KV, rows, n, dtype):
    q, k, v, do = make(rows, H, KV, 40, dtype, seed=rows)
    off = spread(n, rows)
    want = check(q, k, v, do, off)
    out = torch.full((rows + 140, H, 40), 7.0, dtype=dtype, device=DEV)
    assert torch.equal(ops.attention(q, k, v, torch.tensor(off, device=DEV), out=out[:rows]).o, want["o"]) and bool((out[rows:] == 7).all())


@TYPES
def test_a_captured_call_with_room_for_more_sequences(dtype):
    """A graph that is captured for 128 sequences and replayed with fewer, the rest of them empty."""
    H, KV, dim = 6, 2, 64
    q, k, v, do = make(ROWS, H, KV, dim, dtype, seed=5)
    off = torch.full((129,), ROWS, dtype=torch.int64, device=DEV)
    off[:11] = torch.tensor(spread(10))
    o = torch.full((ROWS + 140, H, dim), 7.0, dtype=dtype, device=DEV)

    def call():
        r = ops.attention(q, k, v, off, save=True, out=o[:ROWS])
        return (r.lse,) + ops.attention_backward(q, k, v, off, r.o, r.lse, do)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for n in (10, 63, 128, 1):
        off.fill_(ROWS)
        off[:n + 1] = torch.tensor(spread(n))
        graph.replay()
        got = [o[:ROWS].clone()] + [t.clone() for t in outs]
        want = check(q, k, v, do, spread(n))
        assert all(torch.equal(a, want[name]) for a, name in zip(got, ("o", "lse", "dq", "dk", "dv")))
        assert bool((o[ROWS:] == 7).all())
