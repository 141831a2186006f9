"""CPU-only: outputs and workspaces that lie over other arguments are refused before anything reaches a GPU."""
import ctypes as C
import itertools

from paper_2509_03110_amd import lsam, ops

MB = 1 << 20


def refused(rc, *words):
    return rc == lsam.EINVAL and "lies over" in lsam.last_error() and all(w in lsam.last_error() for w in words)


def test_log_probabilities():
    L = ops._lib()
    d = ops.lsam_logprobs_desc()
    d.rows, d.vocab, d.stride, d.dtype, d.top = 4, 100_000, 100_000, ops.DTYPE_FP32, 5
    need = L.lsam_logprobs_workspace_bytes(C.byref(d))
    assert 0 < need < MB
    names = ["logits", "tokens", "logp", "lse", "entropy", "top_ids", "top_logp", "ws"]
    at = {n: 4 * MB * (i + 1) for i, n in enumerate(names)}

    def forward(n=need, **over):
        a = dict(at, **over)
        return L.lsam_logprobs(C.byref(d), *(a[k] for k in names), n, None)
    assert forward(n=need - 1) == lsam.ENOMEM
    for out, other in itertools.product(["logp", "lse", "entropy", "top_ids", "top_logp"], names[:-1]):
        if out != other:
            assert refused(forward(**{out: at[other] + 4}), out), (out, other)
    for other in names[:-1]:
        assert refused(forward(ws=at[other]), "workspace", other)
    assert refused(forward(ws=at["logits"] + 4 * 399_996 // 16 * 16), "workspace", "logits")

    names = ["logits", "tokens", "lse", "entropy", "g_logp", "g_entropy", "dlogits"]
    at = {n: 4 * MB * (i + 1) for i, n in enumerate(names)}
    for other in names[:-1]:
        a = dict(at, dlogits=at[other] + 4)
        assert refused(L.lsam_logprobs_backward(C.byref(d), *(a[k] for k in names), 100_000, None), "dlogits", other), other
    a = dict(at, dlogits=at["logits"])                       # the logits themselves, but not with another stride
    assert refused(L.lsam_logprobs_backward(C.byref(d), *(a[k] for k in names), 100_001, None), "dlogits")


def test_workspaces_of_recurrences():
    L = ops._lib()
    d = ops.lsam_recurrence_desc()
    d.seqs, d.rows, d.dim, d.dtype, d.packed = 2, 30_000, 10, ops.DTYPE_BF16, 0
    for t in ("f", "x", "h", "dh", "df", "dx"):
        getattr(d, t).stride, getattr(d, t).seq = 10, 300_000
    need = L.lsam_recurrence_workspace_bytes(C.byref(d))
    assert 0 < need < MB
    names = ["f", "x", "h0", "h", "last", "states", "ws"]
    at = {n: 4 * MB * (i + 1) for i, n in enumerate(names)}
    for other in names[:-1]:
        a = dict(at, ws=at[other])
        assert refused(L.lsam_recurrence(C.byref(d), None, *(a[k] for k in names), need, None), "workspace", other)
    names = ["f", "x", "h0", "states", "dh", "dlast", "df", "dx", "dh0", "ws"]
    at = {n: 4 * MB * (i + 1) for i, n in enumerate(names)}
    for other in names[:-1]:
        a = dict(at, ws=at[other])
        assert refused(L.lsam_recurrence_backward(C.byref(d), None, *(a[k] for k in names), need, None), "workspace", other)


def test_workspaces_of_adapters():
    L = ops._lib()
    d = ops.lsam_adapter_desc()
    d.rows, d.in_, d.out, d.rank, d.adapters, d.segs, d.dtype, d.adapter_dtype, d.scale = 100, 32, 48, 8, 3, 4, 1, 0, 1.0
    d.x_stride = d.w_stride = d.a_stride = d.dx_stride = d.da_stride = 32
    d.y_stride = d.dy_stride = 48
    d.b_stride = d.db_stride = 8
    d.a_adapter = d.da_adapter = 8 * 32
    d.b_adapter = d.db_adapter = 8 * 48
    for call, back, names in ((L.lsam_adapter, 0, ["x", "W", "bias", "A", "B", "seg_begin", "seg_adapter", "u", "y"]),
                              (L.lsam_adapter_backward, 1, ["x", "W", "A", "B", "seg_begin", "seg_adapter", "u", "dy", "dx", "dA", "dB"])):
        need = L.lsam_adapter_workspace_bytes(C.byref(d), back)
        assert 0 < need < MB
        at = {n: 4 * MB * (i + 1) for i, n in enumerate(names)}
        for other in names:
            assert refused(call(C.byref(d), *(at[k] for k in names), at[other], need, None), "workspace", other)


# Arrays that go through each other without having a byte in common are two arrays: parts of one wider array, row by row or block by block.
# Whether a call is refused is looked at with a workspace that is too small, or a pointer that is not aligned, which are looked
# for afterwards.

def test_halves_of_one_array_are_no_overlap_for_recurrences():
    L, D = ops._lib(), 10
    for S, T, packed in ((2, 30_000, 0), (1, 60_000, 1)):
        d = ops.lsam_recurrence_desc()
        d.seqs, d.rows, d.dim, d.dtype, d.packed = S, T, D, ops.DTYPE_BF16, packed
        for t in ("f", "x", "h", "dh", "df", "dx"):
            getattr(d, t).stride, getattr(d, t).seq = 2 * D, 2 * D * T
        off = 48 * MB if packed else None

        def forward(h, x):
            return L.lsam_recurrence(C.byref(d), off, 4 * MB, x, None, h, None, None, None, 0, None)

        def backward(df, dx):
            return L.lsam_recurrence_backward(C.byref(d), off, 4 * MB, 4 * MB + 2 * D, None, 20 * MB, 24 * MB, None, df, dx, None, None, 0, None)
        assert forward(8 * MB, 8 * MB + 2 * D) == lsam.ENOMEM and forward(8 * MB + 2 * D, 8 * MB) == lsam.ENOMEM
        assert backward(32 * MB, 32 * MB + 2 * D) == lsam.ENOMEM and backward(32 * MB + 2 * D, 32 * MB) == lsam.ENOMEM
        assert backward(24 * MB + 2 * D, 32 * MB) == lsam.ENOMEM                # beside dh
        assert refused(forward(8 * MB, 8 * MB + 2 * D - 2), "h") and refused(forward(8 * MB, 8 * MB + 2 * D + 2), "h")
        assert refused(backward(32 * MB, 32 * MB + 2 * D + 2), "df")
        d.dx.stride, d.dx.seq = 2 * D + 1, (2 * D + 1) * T                      # rows of other lengths do meet somewhere
        assert refused(backward(32 * MB, 32 * MB + 2 * D), "df")


def test_parts_of_one_array_are_no_overlap_for_adapters_and_dropout():
    L = ops._lib()
    d = ops.lsam_adapter_desc()
    d.rows, d.in_, d.out, d.rank, d.adapters, d.segs, d.dtype, d.adapter_dtype, d.scale = 100, 32, 48, 8, 3, 4, 1, 0, 1.0
    d.x_stride = d.y_stride = d.dx_stride = d.dy_stride = 80                    # x beside y, dx beside dy
    d.w_stride = d.a_stride = 32
    d.b_stride = 8
    d.a_adapter, d.b_adapter = 8 * 32, 8 * 48
    d.da_stride, d.db_stride, d.da_adapter, d.db_adapter = 32, 8, 4000, 2000    # blocks of both fit every 2000
    at = {n: 4 * MB * (i + 1) for i, n in enumerate(["x", "W", "bias", "A", "B", "seg_begin", "seg_adapter", "u", "y", "dy", "dx", "dA", "dB"])}

    def forward(**over):
        a = dict(at, **over)
        return L.lsam_adapter(C.byref(d), *(a[k] for k in ("x", "W", "bias", "A", "B", "seg_begin", "seg_adapter", "u", "y")), None, 0, None)

    def backward(**over):
        a = dict(at, **over)
        return L.lsam_adapter_backward(C.byref(d), *(a[k] for k in ("x", "W", "A", "B", "seg_begin", "seg_adapter", "u", "dy", "dx", "dA", "dB")),
                                       None, 0, None)
    assert forward(y=at["x"] + 64) == lsam.ENOMEM and refused(forward(y=at["x"] + 62), "y") and refused(forward(y=at["x"] + 66), "y")
    assert backward(dx=at["dy"] + 96) == lsam.ENOMEM and refused(backward(dx=at["dy"] + 98), "dx")
    assert backward(dB=at["dA"] + 4 * 256) == lsam.ENOMEM and backward(dB=at["dA"] + 4 * 1616) == lsam.ENOMEM
    assert refused(backward(dB=at["dA"] + 4 * 255), "dA") and refused(backward(dB=at["dA"] + 4 * 1617), "dA")

    p = ops.lsam_dropout_desc()
    p.replicas, p.dtype, p.rows, p.cols, p.p = 2, ops.DTYPE_FP32, 4, 16, 0.5
    p.x_stride = p.y_stride = p.residual_stride = 32
    p.x_replica = p.y_replica = p.residual_replica = 128

    def dropout(x, res, y):
        return L.lsam_dropout(C.byref(p), x, res, y, None)
    assert refused(dropout(4 * MB, None, 4 * MB + 60)) and refused(dropout(4 * MB, None, 4 * MB + 68))
    assert refused(dropout(8 * MB, 4 * MB, 4 * MB + 60))
