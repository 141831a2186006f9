"""CPU-only checks of the operators' boundary: declared symbols are exported and bad arguments are refused on the
host, before anything reaches a GPU."""
import ctypes as C
import os
import re

from paper_2509_03110_amd import lsam, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20           # never dereferenced: the checks fail first, or nothing is to be done


def test_library_exports_every_declared_operator():
    header = open(os.path.join(ROOT, "include", "lsam_ops.h")).read()
    declared = set(re.findall(r"^(?:int|size_t|int64_t) (lsam_[a-z_]+)\s*\(", header, re.M))
    assert declared == set(ops.EXPORTS)
    L = lsam.lib()
    for name in declared:
        assert hasattr(L, name), name


def _dropout(**over):
    d = ops.lsam_dropout_desc()
    d.replicas, d.dtype, d.rows, d.cols, d.p = 2, ops.DTYPE_FP32, 4, 16, 0.5
    d.x_stride = d.y_stride = d.residual_stride = 16
    d.x_replica = d.y_replica = d.residual_replica = 64
    for k, v in over.items():
        setattr(d, k, v)
    return d


def test_dropout_checks_its_arguments_before_touching_the_gpu():
    call = ops._lib().lsam_dropout
    for over, msg in ((dict(dtype=2), "dtype"), (dict(replicas=-1), "replicas"), (dict(replicas=65536), "replicas"),
                      (dict(rows=-1), "rows"), (dict(cols=1 << 31), "cols"), (dict(p=2.0), "p outside"),
                      (dict(p=float("nan")), "p outside"), (dict(site=65536), "site"), (dict(first_replica=65535), "replicas"),
                      (dict(x_stride=15), "stride"), (dict(y_replica=63), "lie over each other"), (dict(x_replica=-1), "stride"),
                      (dict(rows=(1 << 31) - 1, x_stride=1 << 62), "too large")):
        d = _dropout(**over)
        assert call(C.byref(d), FAKE, None, 4 * FAKE, None) == lsam.EINVAL, over
        assert msg in lsam.last_error(), (over, lsam.last_error())
    d = _dropout()
    assert call(None, FAKE, None, FAKE, None) == lsam.EINVAL
    assert call(C.byref(d), None, None, FAKE, None) == lsam.EINVAL
    assert call(C.byref(d), FAKE, None, None, None) == lsam.EINVAL
    assert call(C.byref(d), FAKE, None, FAKE + 4, None) == lsam.EINVAL and "lies over x" in lsam.last_error()
    assert call(C.byref(d), FAKE, 4 * FAKE + 64, 4 * FAKE, None) == lsam.EINVAL and "residual" in lsam.last_error()
    assert call(C.byref(d), FAKE + 2, None, 4 * FAKE, None) == lsam.EINVAL and "aligned" in lsam.last_error()
    for over in (dict(rows=0), dict(cols=0), dict(replicas=0)):
        assert call(C.byref(_dropout(**over)), None, None, None, None) == 0


def test_logprobs_checks_its_arguments_before_touching_the_gpu():
    L = ops._lib()

    def desc(**over):
        d = ops.lsam_logprobs_desc()
        d.rows, d.vocab, d.stride, d.dtype, d.top = 4, 1000, 1000, ops.DTYPE_BF16, 5
        for k, v in over.items():
            setattr(d, k, v)
        return C.byref(d)
    for over, msg in ((dict(dtype=5), "dtype"), (dict(rows=-1), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=1 << 31), "vocab"),
                      (dict(top=33), "top"), (dict(top=-1), "top"), (dict(vocab=4, top=5), "top"), (dict(stride=999), "stride"),
                      (dict(rows=1 << 40, stride=1 << 40), "too large")):
        assert L.lsam_logprobs(desc(**over), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, None) == lsam.EINVAL, over
        assert msg in lsam.last_error(), (over, lsam.last_error())
        assert L.lsam_logprobs_workspace_bytes(desc(**over)) == 0
        assert L.lsam_logprobs_backward(desc(**over), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 8 * FAKE, 1000, None) == lsam.EINVAL, over
    need = L.lsam_logprobs_workspace_bytes(desc(vocab=100_000, stride=100_000))
    assert need > 0 and L.lsam_logprobs_workspace_bytes(desc()) == 0 and L.lsam_logprobs_workspace_bytes(desc(rows=5000)) == 0
    big = desc(vocab=100_000, stride=100_000)
    assert L.lsam_logprobs(big, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need - 1, None) == lsam.ENOMEM
    assert L.lsam_logprobs(big, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, need, None) == lsam.ENOMEM
    assert L.lsam_logprobs(big, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE + 8, need, None) == lsam.EINVAL
    assert L.lsam_logprobs(desc(), None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, None) == lsam.EINVAL
    assert L.lsam_logprobs(desc(), FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, None, 0, None) == lsam.EINVAL
    assert L.lsam_logprobs(desc(), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, None, 0, None) == lsam.EINVAL
    assert L.lsam_logprobs(desc(), FAKE + 1, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, 0, None) == lsam.EINVAL
    assert L.lsam_logprobs_backward(desc(), FAKE, None, FAKE, FAKE, FAKE, FAKE, 8 * FAKE, 1000, None) == lsam.EINVAL
    assert L.lsam_logprobs_backward(desc(), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE + 16, 1000, None) == lsam.EINVAL
    assert L.lsam_logprobs_backward(desc(), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 8 * FAKE, 999, None) == lsam.EINVAL
    assert L.lsam_logprobs(desc(rows=0), None, None, None, None, None, None, None, None, 0, None) == 0
    assert L.lsam_logprobs_backward(desc(rows=0), None, None, None, None, None, None, None, 1000, None) == 0


def test_recurrence_checks_its_arguments_before_touching_the_gpu():
    L = ops._lib()

    def desc(**over):
        d = ops.lsam_recurrence_desc()
        d.seqs, d.rows, d.dim, d.dtype, d.packed = 2, 30, 10, ops.DTYPE_FP32, 0
        for t in ("f", "x", "h", "dh", "df", "dx"):
            getattr(d, t).stride, getattr(d, t).seq = 10, 300
        for k, v in over.items():
            if k.endswith("_seq") or k.endswith("_stride"):
                setattr(getattr(d, k.split("_")[0]), k.split("_")[1], v)
            else:
                setattr(d, k, v)
        return C.byref(d)
    P = [FAKE * k for k in range(1, 13)]

    def forward(d, off=None, f=P[0], x=P[1], h0=None, h=P[2], last=P[3], states=P[4], ws=None, n=0):
        return L.lsam_recurrence(d, off, f, x, h0, h, last, states, ws, n, None)

    def backward(d, off=None, f=P[0], x=P[1], h0=None, states=P[4], dh=P[5], dlast=None, df=P[6], dx=P[7], dh0=P[8], ws=None, n=0):
        return L.lsam_recurrence_backward(d, off, f, x, h0, states, dh, dlast, df, dx, dh0, ws, n, None)
    for over, msg in ((dict(dtype=-1), "dtype"), (dict(packed=2), "packed"), (dict(seqs=-1), "seqs"), (dict(rows=-1), "rows"),
                      (dict(dim=0), "dim"), (dict(rows=1 << 39, seqs=1 << 30), "too large"), (dict(seqs=1 << 30, dim=1 << 20), "too large"),
                      (dict(f_stride=9), "stride of f"), (dict(x_seq=-1), "stride of x")):
        assert forward(desc(**over)) == lsam.EINVAL and msg in lsam.last_error(), (over, lsam.last_error())
        assert backward(desc(**over)) == lsam.EINVAL and msg in lsam.last_error(), (over, lsam.last_error())
    assert forward(desc(h_seq=299)) == lsam.EINVAL and "stride of h" in lsam.last_error()
    assert backward(desc(df_seq=5)) == lsam.EINVAL and "stride of df" in lsam.last_error()
    assert forward(desc(packed=1)) == lsam.EINVAL and "offsets" in lsam.last_error()
    assert forward(desc(), h=P[1]) == lsam.EINVAL and "lies over" in lsam.last_error()
    assert forward(desc(), last=P[4] + 40) == lsam.EINVAL and "lies over" in lsam.last_error()
    assert forward(desc(), f=None) == lsam.EINVAL and forward(desc(), h=None) == lsam.EINVAL
    assert forward(desc(), h0=FAKE + 2) == lsam.EINVAL and "aligned" in lsam.last_error()
    assert backward(desc(), states=None) == lsam.EINVAL and backward(desc(), dx=P[6]) == lsam.EINVAL
    long = desc(rows=100_000, f_seq=1 << 20, x_seq=1 << 20, h_seq=1 << 20, dh_seq=1 << 20, df_seq=1 << 20, dx_seq=1 << 20)
    need = L.lsam_recurrence_workspace_bytes(long)
    far = dict(f=1 << 30, x=2 << 30, h=3 << 30, last=4 << 30, states=5 << 30)
    assert need > 0 and L.lsam_recurrence_workspace_bytes(desc()) == 0
    assert forward(long, **far) == lsam.ENOMEM and forward(long, ws=6 << 30, n=need - 1, **far) == lsam.ENOMEM
    assert forward(long, ws=(6 << 30) + 4, n=need, **far) == lsam.EINVAL
    assert L.lsam_recurrence_states(desc()) == 2 and L.lsam_recurrence_states(desc(dim=0)) == lsam.EINVAL
    assert forward(desc(seqs=0), f=None, x=None, h=None) == 0 and backward(desc(seqs=0), f=None) == 0


def test_adapter_checks_its_arguments_before_touching_the_gpu():
    L = ops._lib()

    def desc(**over):
        d = ops.lsam_adapter_desc()
        d.rows, d.in_, d.out, d.rank, d.adapters, d.segs, d.dtype, d.adapter_dtype, d.scale = 100, 32, 48, 8, 3, 4, 1, 0, 1.0
        d.x_stride = d.w_stride = d.a_stride = d.dx_stride = d.da_stride = 32
        d.y_stride = d.dy_stride = 48
        d.b_stride = d.db_stride = 8
        d.a_adapter = d.da_adapter = 8 * 32
        d.b_adapter = d.db_adapter = 8 * 48
        for k, v in over.items():
            setattr(d, k, v)
        return C.byref(d)
    P = {n: FAKE * (i + 1) for i, n in enumerate(("x", "W", "bias", "A", "B", "begin", "which", "u", "y", "dy", "dx", "dA", "dB", "ws"))}

    def forward(d, n=1 << 20, **over):
        a = dict(P, **over)
        return L.lsam_adapter(d, *(a[k] for k in ("x", "W", "bias", "A", "B", "begin", "which", "u", "y", "ws")), n, None)

    def backward(d, n=1 << 20, **over):
        a = dict(P, **over)
        return L.lsam_adapter_backward(d, *(a[k] for k in ("x", "W", "A", "B", "begin", "which", "u", "dy", "dx", "dA", "dB", "ws")), n, None)
    for over, msg in ((dict(dtype=2), "dtype"), (dict(adapter_dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 28), "rows"),
                      (dict(in_=0), "in and out"), (dict(out=(1 << 21) + 1), "in and out"), (dict(rank=0), "rank"), (dict(rank=65), "rank"),
                      (dict(adapters=-1), "adapters"), (dict(adapters=65536), "adapters"), (dict(segs=-1), "segs"),
                      (dict(in_=1 << 20, out=1 << 20), "too large"), (dict(rows=1 << 27, in_=1 << 20), "too large"),
                      (dict(x_stride=31), "stride of x"), (dict(w_stride=-32), "stride of W"), (dict(a_stride=31), "stride of A"),
                      (dict(b_adapter=-1), "stride of B")):
        assert forward(desc(**over)) == lsam.EINVAL and msg in lsam.last_error(), (over, lsam.last_error())
        assert backward(desc(**over)) == lsam.EINVAL and msg in lsam.last_error(), (over, lsam.last_error())
    assert forward(desc(y_stride=47)) == lsam.EINVAL and backward(desc(dy_stride=47)) == lsam.EINVAL
    assert backward(desc(dx_stride=31)) == lsam.EINVAL and backward(desc(da_adapter=255)) == lsam.EINVAL
    assert backward(desc(db_stride=7)) == lsam.EINVAL
    for name in ("x", "W", "A", "B", "begin", "which", "u", "y"):
        assert forward(desc(), **{name: None}) == lsam.EINVAL and "NULL" in lsam.last_error(), (name, lsam.last_error())
    for name in ("x", "W", "A", "B", "begin", "which", "u", "dy"):
        assert backward(desc(), **{name: None}) == lsam.EINVAL and "NULL" in lsam.last_error(), (name, lsam.last_error())
    assert backward(desc(), dA=None) == lsam.EINVAL and "together" in lsam.last_error()
    assert forward(desc(), y=P["x"]) == lsam.EINVAL and "lies over" in lsam.last_error()
    assert backward(desc(), dx=P["dy"] + 2) == lsam.EINVAL and "lies over" in lsam.last_error()
    assert backward(desc(), dB=P["dA"] + 64) == lsam.EINVAL and "lies over" in lsam.last_error()
    # blocks of one array per adapter, in turn: dB may not reach into dA's blocks
    apart = desc(da_adapter=1000, db_adapter=1000)
    assert backward(apart, dB=P["dA"] + 4 * 255) == lsam.EINVAL and "lies over" in lsam.last_error()
    assert backward(apart, dB=P["dA"] + 4 * 617) == lsam.EINVAL and "lies over" in lsam.last_error()
    assert backward(apart, dB=P["dA"] + 4 * 616, n=0) == lsam.ENOMEM
    assert forward(desc(), x=P["x"] + 1) == lsam.EINVAL and "aligned" in lsam.last_error()
    assert forward(desc(), ws=None) == lsam.ENOMEM and forward(desc(), ws=P["ws"] + 16) == lsam.EINVAL
    assert L.lsam_adapter_workspace_bytes(desc(rank=0), 0) == 0 and L.lsam_adapter_workspace_bytes(desc(rows=64), 0) == 256
    assert L.lsam_adapter_workspace_bytes(desc(), 1) > 100 * 8 * 4
    assert forward(desc(rows=0), x=None, y=None, u=None) == 0
