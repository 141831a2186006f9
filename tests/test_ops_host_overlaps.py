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
