"""Sizes that take each branch of the operators' plans, against the definitions and with the bounds of their own test files."""
import pytest
import torch

import test_gpu_adapter as adapter
import test_gpu_recurrence as recurrence

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# Packed sequences of 16 rows or less on the average: one wavefront a workgroup, in tiles of 16 rows, of which a long sequence has several.
@pytest.mark.parametrize("dtype", [recurrence.F32, recurrence.B16])
@pytest.mark.parametrize("D,lengths", [
    (5, [1] * 9 + [121]),                                   # cut into runs
    (70, [3, 0, 1, 150, 0, 2, 1, 1, 1, 33, 2, 0, 17, 1, 1, 5]),
    (130, [1] * 60 + [900] + [2] * 40),                     # workgroups enough without
    (1, [0, 2] * 130 + [1300] + [1] * 15)])
def test_one_wavefront_over_several_tiles(dtype, D, lengths):
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    assert offsets[-1] <= 16 * len(lengths) and max(lengths) > 100
    f, x, h0, dh, dlast = recurrence.make((offsets[-1], D), len(lengths), dtype, seed=D)
    recurrence.check(f, x, h0, dh, dlast, torch.tensor(offsets, dtype=torch.int64, device=DEV))


# Rank-sized products in tiles of 32 rows (6144 to 7167 rows) and of 64; rows that go to LDS as they lie, and others.
@pytest.mark.parametrize("dtype,atype", adapter.TYPES)
@pytest.mark.parametrize("rows", [6200, 7300])
@pytest.mark.parametrize("inp,out", [(72, 40), (71, 41)])
@pytest.mark.parametrize("rank", [8, 24, 64])
def test_rank_sized_products_in_larger_tiles(dtype, atype, rows, inp, out, rank):
    x, W, A, B, bias, dy = adapter.make(rows, inp, out, rank, 3, dtype, atype, seed=rows + rank)
    adapter.check(x, W, A, B, bias, dy, [0, 100, 101, 3000, 3000, rows - 5], [2, -1, 0, 1, 0])


# At most 64 rows of many outputs, whose adapters' copies would serve few rows each.
@pytest.mark.parametrize("rows,segs", [(1, 1), (16, 5), (40, 40), (64, 17)])
def test_few_rows_of_many_adapters_and_outputs(rows, segs):
    begin = [rows * k // segs for k in range(segs)] + [rows]
    x, W, A, B, bias, dy = adapter.make(rows, 48, 8400, 12, segs, adapter.B16, adapter.B16, seed=rows)
    adapter.check(x, W, A, B, bias, dy, begin, list(range(segs)))
