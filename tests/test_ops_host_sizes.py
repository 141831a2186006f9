"""CPU-only: what the operators ask for goes by what a call uses."""
import ctypes as C

from paper_2509_03110_amd import ops


def adapter(rows, inp, out, rank, adapters, segs, dtype=ops.DTYPE_BF16):
    d = ops.lsam_adapter_desc()
    d.rows, d.in_, d.out, d.rank, d.adapters, d.segs = rows, inp, out, rank, adapters, segs
    d.dtype, d.adapter_dtype, d.scale = dtype, dtype, 1.0
    return C.byref(d)


def test_an_adapter_calls_workspace_goes_by_its_segments_not_by_adapters_it_does_not_use():
    need = ops._lib().lsam_adapter_workspace_bytes
    for rows in (65, 2000):
        for back in (0, 1):
            four = need(adapter(rows, 4096, 4096, 16, 4, 4), back)
            assert need(adapter(rows, 4096, 4096, 16, 1000, 4), back) == four
            assert need(adapter(rows, 4096, 4096, 16, 4, 1000), back) == four
            assert need(adapter(rows, 4096, 4096, 16, 1000, 0), back) < four
    # a token: no copy of what it does not need is larger than the matrix itself
    for rank, adapters in ((64, 256), (16, 1000)):
        assert need(adapter(1, 4096, 14336, rank, adapters, 1), 0) < 4096 * 14336 * 2
        assert need(adapter(64, 4096, 14336, rank, adapters, 64), 0) < 4096 * 14336 * 2
