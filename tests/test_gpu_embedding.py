"""lsam_embedding and its gradient against the definition in 64 bits.

Tolerances (u = 2^-24): a row of y is one product in fp32 (u of itself) and, stored in bfloat16, a rounding by 2^-8 of itself.  A row of the
gradient is a sum of n numbers in fp32, each of which passes at most n additions, and one product: (n + 1) u of the sum of absolute
values, and u of the sum itself for the product's operand.  Sums of small whole numbers times a power of two are exact."""
import math

import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, B16 = torch.float32, torch.bfloat16


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def some_tokens(K, rows, V, seed, hot=0.3):
    """Most of them any, some one and the same, some that hold nothing."""
    g = gen(seed)
    t = torch.randint(0, V, (K, rows), device=DEV, generator=g, dtype=torch.int32)
    t[torch.rand(K, rows, device=DEV, generator=g) < hot] = V // 2
    pad = torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    hole = torch.rand(K, rows, device=DEV, generator=g) < 0.1
    t[hole] = pad[torch.randint(0, 4, (int(hole.sum()),), device=DEV, generator=g)]
    return t


def check_lookup(y, tokens, table, scale):
    K, rows = tokens.shape
    table = table.expand(K, *table.shape[-2:]).double()
    there = (tokens >= 0) & (tokens < table.shape[1])
    want = torch.stack([table[k][tokens[k].long().clamp(0, table.shape[1] - 1)] for k in range(K)]) * scale * there[:, :, None]
    tol = (U + (2.0 ** -8 if y.dtype == B16 else 0)) * want.abs()
    assert bool(((y.double() - want).abs() <= tol).all())


def check_gradient(d, tokens, dy, scale):
    K, rows = tokens.shape
    V = d.shape[1]
    for k in range(K):
        keep = (tokens[k] >= 0) & (tokens[k] < V)
        t, g = tokens[k][keep].long(), dy[k][keep].double()
        zero = torch.zeros(V, dy.shape[2], dtype=torch.float64, device=DEV)
        want, size = zero.index_add(0, t, g) * scale, zero.index_add(0, t, g.abs()) * abs(scale)
        n = torch.bincount(t, minlength=V)[:, None]
        assert bool(((d[k].double() - want).abs() <= (n + 2) * U * size).all())


SIZES = [(1, 1, 1, 1), (1, 63, 5, 3), (2, 64, 7, 4), (1, 65, 1000, 257), (3, 1000, 13, 33), (1, 5000, 2, 8), (2, 3000, 3000, 256),
         (1, 700, 200001, 5), (2, 129, 600, 260), (5, 200, 1, 1030), (1, 20001, 300, 3), (2, 33000, 1500, 6)]   # the last two: places in parts


@pytest.mark.parametrize("K,rows,V,D", SIZES)
@pytest.mark.parametrize("table_type,dtype", [(F32, F32), (F32, B16), (B16, B16), (B16, F32)])
def test_lookup_and_gradient(K, rows, V, D, table_type, dtype):
    g = gen(rows + D)
    tokens = some_tokens(K, rows, V, seed=rows)
    table = torch.randn(K, V, D, device=DEV, generator=g).to(table_type)
    dy = torch.randn(K, rows, D, device=DEV, generator=g).to(dtype)
    y = ops.embedding(tokens, table, scale=1.3125, dtype=dtype)
    assert y.dtype == dtype
    check_lookup(y, tokens, table, 1.3125)
    d = ops.embedding_backward(tokens, dy, V, scale=1.3125)
    check_gradient(d, tokens, dy, 1.3125)
    assert torch.equal(d, ops.embedding_backward(tokens, dy, V, scale=1.3125))
    whole = torch.randint(-3, 4, dy.shape, device=DEV, generator=g)
    got = ops.embedding_backward(tokens, whole.to(dtype), V, scale=0.5)
    for k in range(K):
        keep = (tokens[k] >= 0) & (tokens[k] < V)
        want = torch.zeros(V, D, dtype=torch.int64, device=DEV).index_add_(0, tokens[k][keep].long(), whole[k][keep])
        assert torch.equal(got[k], want.float() * 0.5)


@pytest.mark.parametrize("tokens", [[0] * 64, [3] * 128 + [1], [1] * 63 + [2] * 66, [2] * 64 + [1] * 64 + [0] * 64, [-1] * 70, [4, -1] * 200 + [0] * 65])
def test_tokens_that_end_at_and_beside_the_edges_of_64_places(tokens):
    t = torch.tensor([tokens], dtype=torch.int32, device=DEV)
    dy = torch.randint(-8, 9, (1, len(tokens), 6), device=DEV, generator=gen(1)).float()
    got = ops.embedding_backward(t, dy, 5)
    keep = t[0] >= 0
    assert torch.equal(got[0], torch.zeros(5, 6, device=DEV).index_add_(0, t[0][keep].long(), dy[0][keep]))


@pytest.mark.parametrize("before", [0, 1, 63])
@pytest.mark.parametrize("n", [64 * 8, 64 * 9, 64 * 9 + 1, 64 * 10 - 1, 64 * 70 + 5])
def test_runs_over_few_and_many_chunks_of_64_places(n, before):
    """One token's run, and a shorter one behind it, with columns for three wavefronts; small whole numbers, so exact."""
    t = torch.tensor([[0] * before + [1] * n + [2] * 200], dtype=torch.int32, device=DEV)
    t = t[:, torch.randperm(t.shape[1], device=DEV, generator=gen(n))].contiguous()
    dy = torch.randint(-8, 9, (1, t.shape[1], 520), device=DEV, generator=gen(1)).float()
    assert torch.equal(ops.embedding_backward(t, dy, 4)[0], torch.zeros(4, 520, device=DEV).index_add_(0, t[0].long(), dy[0]))


@pytest.mark.parametrize("table_type,dtype,rows,D", [(F32, F32, 22000, 777), (B16, F32, 33000, 513), (F32, B16, 33000, 1031), (B16, B16, 60000, 600)])
def test_many_rows_of_which_a_lane_has_several(table_type, dtype, rows, D):
    tokens = some_tokens(2, rows, 50, seed=rows)
    wide = torch.full((2, rows, D + 5), 7.0, dtype=dtype, device=DEV)
    table = torch.randn(2, 50, D, device=DEV, generator=gen(5)).to(table_type)
    y = ops.embedding(tokens, table, scale=0.75, out=wide[:, :, 3:3 + D])
    there = (tokens >= 0) & (tokens < 50)
    for k in range(2):
        want = (table[k].float() * 0.75).to(dtype)[tokens[k].long().clamp(0, 49)]          # one product, one rounding: exact
        assert torch.equal(y[k], torch.where(there[k][:, None], want, torch.zeros_like(want)))
    assert bool((wide[:, :, :3] == 7).all()) and bool((wide[:, :, 3 + D:] == 7).all())


def test_one_replica_without_its_index_and_a_table_that_all_read():
    tokens = some_tokens(3, 50, 20, seed=2)
    table = torch.randn(20, 12, device=DEV, generator=gen(3))
    check_lookup(ops.embedding(tokens, table, scale=2.0), tokens, table, 2.0)
    assert torch.equal(ops.embedding(tokens[1], table), ops.embedding(tokens, table)[1])
    dy = torch.randn(3, 50, 12, device=DEV, generator=gen(4))
    shared = ops.embedding_backward(tokens.view(-1), dy.view(-1, 12), 20)
    check_gradient(shared[None], tokens.view(1, -1), dy.view(1, -1, 12), 1.0)


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("pad", [1, 4])
def test_parts_of_wider_arrays_and_of_rows_of_parameters(dtype, pad):
    K, rows, V, D = 2, 300, 40, 21
    g = gen(5)
    tokens = torch.randint(0, V, (K, rows + 7), device=DEV, generator=g, dtype=torch.int32)[:, 3:3 + rows]
    params = torch.randn(K, 1000, device=DEV, generator=g)
    table = params.as_strided((K, V, D), (1000, D, 1), 5)
    wide = torch.full((K, rows, D + 2 * pad), 7.0, device=DEV, dtype=dtype)
    y = ops.embedding(tokens, table, scale=0.5, out=wide[:, :, pad:pad + D])
    check_lookup(y, tokens, table, 0.5)
    assert bool((wide[:, :, :pad] == 7).all()) and bool((wide[:, :, pad + D:] == 7).all())
    dy = torch.randn(K, rows, D + pad, device=DEV, generator=g).to(dtype)[:, :, pad:]
    grads = torch.full((K, 1000), 9.0, device=DEV)
    ops.embedding_backward(tokens, dy, V, scale=0.5, out=grads.as_strided((K, V, D), (1000, D, 1), 5))
    check_gradient(grads[:, 5:5 + V * D].reshape(K, V, D), tokens, dy, 0.5)
    assert bool((grads[:, :5] == 9).all()) and bool((grads[:, 5 + V * D:] == 9).all())


def test_rows_that_hold_nothing_reach_nothing():
    tokens = torch.tensor([[2, -1, 0, 5, 2]], dtype=torch.int32, device=DEV)
    table = torch.randn(1, 5, 9, device=DEV)
    table[0, 1] = math.nan                                            # a row that no token names
    y = ops.embedding(tokens, table)
    assert bool((y[0, [1, 3]] == 0).all()) and bool(y.isfinite().all())
    dy = torch.randn(1, 5, 9, device=DEV)
    dy[0, [1, 3]] = math.nan
    d = ops.embedding_backward(tokens, dy, 5)
    assert bool(d.isfinite().all()) and torch.equal(d[0, 2], dy[0, 0] + dy[0, 4]) and bool((d[0, [1, 3, 4]] == 0).all())


def test_no_rows_and_no_replicas():
    none = torch.empty(2, 0, dtype=torch.int32, device=DEV)
    assert ops.embedding(none, torch.randn(2, 4, 8, device=DEV)).shape == (2, 0, 8)
    assert torch.equal(ops.embedding_backward(none, torch.empty(2, 0, 8, device=DEV), 4), torch.zeros(2, 4, 8, device=DEV))
    assert ops.embedding_backward(none[:0], torch.empty(0, 0, 8, device=DEV), 4).shape == (0, 4, 8)


def test_refusals():
    t, table = torch.zeros(2, 5, dtype=torch.int32, device=DEV), torch.randn(2, 4, 8, device=DEV)
    dy = torch.randn(2, 5, 8, device=DEV)
    for call, word in [(lambda: ops.embedding(t.long(), table), "int32"), (lambda: ops.embedding(t, table[:1]), "shape"),
                       (lambda: ops.embedding(t[0], table), "indices"), (lambda: ops.embedding(t, table.half()), "bfloat16"),
                       (lambda: ops.embedding(t, table.transpose(1, 2)), "contiguous"), (lambda: ops.embedding(t.cpu(), table), "GPU"),
                       (lambda: ops.embedding(t, table, out=dy[:, :, :4]), "shape"), (lambda: ops.embedding(t, table, dtype=B16, out=dy), "bfloat16"),
                       (lambda: ops.embedding_backward(t, dy[0], 4), "indices"), (lambda: ops.embedding_backward(t, dy, 0), "vocab"),
                       (lambda: ops.embedding_backward(t, dy, ops.EMBEDDING_MAX_VOCAB + 1), "vocab"),
                       (lambda: ops.embedding(t, table.requires_grad_()), "gradient")]:
        with pytest.raises(lsam.LsamError) as e:
            call()
        assert e.value.code == lsam.EINVAL and word in str(e.value), (word, str(e.value))
