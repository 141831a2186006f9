"""ctypes binding of the operators in include/lsam_ops.h: argument marshalling only.

Tensors are checked for what the C boundary cannot see (device, type, shape, contiguous last index) and handed over
as they lie, strides included.  Outputs that are not given are allocated on the stream that the call runs on: the
current stream of x's device, or `stream` (a torch.cuda.Stream).  As with any torch operation, inputs that were made
on another stream have to be ready on this one, and tensors that are dropped while another stream still reads them
need record_stream.  Gradients are entry points of their own; nothing here records for autograd, and tensors that require
a gradient are refused while torch records (torch.no_grad(), or detach() them).
"""
from __future__ import annotations

import ctypes as C
from collections import namedtuple

from . import lsam
from .lsam import EINVAL, LsamError

DTYPE_FP32, DTYPE_BF16 = 0, 1

TOP_MAX = 32
ADAPTER_MAX_RANK = 64

EXPORTS = ["lsam_dropout", "lsam_logprobs_workspace_bytes", "lsam_logprobs", "lsam_logprobs_backward",
           "lsam_recurrence_workspace_bytes", "lsam_recurrence_states", "lsam_recurrence", "lsam_recurrence_backward",
           "lsam_adapter_workspace_bytes", "lsam_adapter", "lsam_adapter_backward"]


class lsam_dropout_desc(C.Structure):
    _fields_ = [
        ("replicas", C.c_int32), ("dtype", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64),
        ("x_stride", C.c_int64), ("x_replica", C.c_int64),
        ("residual_stride", C.c_int64), ("residual_replica", C.c_int64),
        ("y_stride", C.c_int64), ("y_replica", C.c_int64),
        ("p", C.c_double), ("seed", C.c_uint64), ("step", C.c_uint32), ("site", C.c_uint32),
        ("first_replica", C.c_uint32),
    ]


class lsam_logprobs_desc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int64), ("stride", C.c_int64), ("dtype", C.c_int32), ("top", C.c_int32)]


class lsam_rows(C.Structure):
    _fields_ = [("stride", C.c_int64), ("seq", C.c_int64)]


class lsam_recurrence_desc(C.Structure):
    _fields_ = [("seqs", C.c_int64), ("rows", C.c_int64), ("dim", C.c_int64), ("dtype", C.c_int32), ("packed", C.c_int32),
                ("f", lsam_rows), ("x", lsam_rows), ("h", lsam_rows), ("dh", lsam_rows), ("df", lsam_rows), ("dx", lsam_rows)]


class lsam_adapter_desc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("in_", C.c_int32), ("out", C.c_int32), ("rank", C.c_int32), ("adapters", C.c_int32),
                ("segs", C.c_int32), ("dtype", C.c_int32), ("adapter_dtype", C.c_int32), ("scale", C.c_float)] + [
                    (n, C.c_int64) for n in ("x_stride", "w_stride", "y_stride", "a_adapter", "a_stride", "b_adapter", "b_stride",
                                             "dy_stride", "dx_stride", "da_adapter", "da_stride", "db_adapter", "db_stride")]


_ready = None
torch = None              # imported with the library's first use, as in lsam.py


def _lib():
    global _ready, torch
    if _ready is None:
        import torch
        L = lsam.lib()
        vp = C.c_void_p
        L.lsam_dropout.restype = C.c_int
        L.lsam_dropout.argtypes = [C.POINTER(lsam_dropout_desc), vp, vp, vp, vp]
        L.lsam_logprobs_workspace_bytes.restype = C.c_size_t
        L.lsam_logprobs_workspace_bytes.argtypes = [C.POINTER(lsam_logprobs_desc)]
        L.lsam_logprobs.restype = C.c_int
        L.lsam_logprobs.argtypes = [C.POINTER(lsam_logprobs_desc)] + [vp] * 8 + [C.c_size_t, vp]
        L.lsam_logprobs_backward.restype = C.c_int
        L.lsam_logprobs_backward.argtypes = [C.POINTER(lsam_logprobs_desc)] + [vp] * 7 + [C.c_int64, vp]
        rec = C.POINTER(lsam_recurrence_desc)
        L.lsam_recurrence_workspace_bytes.restype = C.c_size_t
        L.lsam_recurrence_workspace_bytes.argtypes = [rec]
        L.lsam_recurrence_states.restype = C.c_int64
        L.lsam_recurrence_states.argtypes = [rec]
        L.lsam_recurrence.restype = C.c_int
        L.lsam_recurrence.argtypes = [rec] + [vp] * 8 + [C.c_size_t, vp]
        L.lsam_recurrence_backward.restype = C.c_int
        L.lsam_recurrence_backward.argtypes = [rec] + [vp] * 11 + [C.c_size_t, vp]
        L.lsam_adapter_workspace_bytes.restype = C.c_size_t
        L.lsam_adapter_workspace_bytes.argtypes = [C.POINTER(lsam_adapter_desc), C.c_int32]
        L.lsam_adapter.restype = C.c_int
        L.lsam_adapter.argtypes = [C.POINTER(lsam_adapter_desc)] + [vp] * 10 + [C.c_size_t, vp]
        L.lsam_adapter_backward.restype = C.c_int
        L.lsam_adapter_backward.argtypes = [C.POINTER(lsam_adapter_desc)] + [vp] * 12 + [C.c_size_t, vp]
        _ready = L
    return _ready


def _check(rc):
    if rc < 0:
        raise LsamError(rc, lsam.last_error())
    return rc


def _refuse(msg):
    raise LsamError(EINVAL, msg)


def _dtype(t, what):
    if t.dtype == torch.float32:
        return DTYPE_FP32
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    _refuse("%s is %s: float32 or bfloat16 is wanted" % (what, t.dtype))


def _expect(t, what, like=None, shape=None, dtype=None, dense=False):
    """Whether `t` is a tensor of that device, shape and type with a contiguous last index (dense: all of it)."""
    if not t.is_cuda:
        _refuse("%s is not on a GPU" % what)
    if t.requires_grad and torch.is_grad_enabled():
        _refuse("%s requires a gradient, which this call does not record: see its backward call, and torch.no_grad()" % what)
    if like is not None and t.device != like.device:
        _refuse("%s is on %s, not on %s" % (what, t.device, like.device))
    if shape is not None and t.shape != shape:
        _refuse("%s has shape %s: %s is wanted" % (what, tuple(t.shape), tuple(shape)))
    if dtype is not None and t.dtype != dtype:
        _refuse("%s is %s: %s is wanted" % (what, t.dtype, dtype))
    if t.is_contiguous():
        return
    if dense:
        _refuse("%s must be contiguous" % what)
    if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("the last index of %s must be contiguous" % what)


class _On:
    """The device and stream that a call runs on, current while it lasts; entered, the stream's handle."""
    __slots__ = ("device", "context")

    def __init__(self, t, stream):
        self.device, self.context = t.device, None
        if stream is not None:
            if stream.device != t.device:
                _refuse("the stream belongs to %s, the tensors to %s" % (stream.device, t.device))
            self.context = torch.cuda.stream(stream)
        elif torch.cuda.current_device() != t.device.index:
            self.context = torch.cuda.device(t.device)

    def __enter__(self):
        if self.context is not None:
            self.context.__enter__()
        return _raw_stream(self.device.index)

    def __exit__(self, *err):
        if self.context is not None:
            self.context.__exit__(*err)


def _raw_stream(index):
    """Handle of the device's current stream.  (A Stream object for it costs 2 us, a third of a small call.)"""
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(index) if get is not None else torch.cuda.current_stream(index).cuda_stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def dropout(x, p, seed, step, site=0, first_replica=0, residual=None, out=None, stream=None):
    """residual + m x / (1 - p) with the mask m of (seed, step, site, place); see lsam_dropout.  x: [K, rows, cols]
    of K replicas, [rows, cols] or [cols] of one.  The gradient of x is the same call on the gradient of the result,
    with no residual.  `out` may be x or the residual."""
    call = (_ready or _lib()).lsam_dropout
    n = x.dim()
    if not 1 <= n <= 3:
        _refuse("x has %d indices: 1 to 3 are wanted" % n)
    _expect(x, "x")
    if residual is not None:
        _expect(residual, "the residual", x, x.shape, x.dtype)
    if out is not None:
        _expect(out, "out", x, x.shape, x.dtype)
    if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 32 and 0 <= site < 1 << 16 and 0 <= first_replica < 1 << 16):
        _refuse("the seed has 64 bits, the step 32, the site and the replica 16")
    lead = (1,) * (3 - n)
    none = (0,) * (3 - n)
    with _On(x, stream) as raw:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        K, rows, cols = lead + x.shape
        xk, xr, _ = none + x.stride()
        yk, yr, _ = none + y.stride()
        rk, rr, _ = none + residual.stride() if residual is not None else (0, 0, 0)
        d = lsam_dropout_desc(K, _dtype(x, "x"), rows, cols, xr, xk, rr, rk, yr, yk, p, seed, step, site, first_replica)
        _check(call(C.byref(d), x.data_ptr(), _ptr(residual), y.data_ptr(), raw))
    return y



LogProbs = namedtuple("LogProbs", "logp lse entropy top_ids top_logp")


def _logprobs_desc(logits, top):
    if logits.dim() != 2:
        _refuse("the logits have %d indices: [rows, vocab] is wanted" % logits.dim())
    _expect(logits, "logits")
    rows, vocab = logits.shape
    return lsam_logprobs_desc(rows, vocab, logits.stride(0), _dtype(logits, "logits"), top)


def logprobs(logits, tokens=None, top=0, stream=None):
    """Log probabilities of tokens [rows] (int32; one outside the vocabulary does not count: 0) under logits
    [rows, vocab], with the log normaliser in two parts lse [rows, 2] (the largest logit m, and ln sum e^{z - m}), the
    entropy [rows], and the `top` largest logits' indices and log probabilities [rows, top]; see lsam_logprobs.  Fields that were not asked for
    are None."""
    L = _ready or _lib()
    if not 0 <= top <= TOP_MAX:
        _refuse("top is %d: 0 to %d are possible" % (top, TOP_MAX))
    d = _logprobs_desc(logits, top)
    rows = logits.shape[0]
    if tokens is not None:
        _expect(tokens, "tokens", logits, (rows,), torch.int32, True)
    at = C.byref(d)
    with _On(logits, stream) as raw:
        need = L.lsam_logprobs_workspace_bytes(at)
        device = logits.device
        # one allocation for the columns of numbers
        logp, entropy, lse, best = torch.empty(rows * (4 + top), dtype=torch.float32, device=device).split_with_sizes(
            (rows, rows, 2 * rows, rows * top))
        lse = lse.view(rows, 2)
        ids = None
        if top > 0:
            best = best.view(rows, top)
            ids = torch.empty((rows, top), dtype=torch.int32, device=device)
        ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        _check(L.lsam_logprobs(at, logits.data_ptr(), _ptr(tokens), logp.data_ptr(), lse.data_ptr(), entropy.data_ptr(), _ptr(ids),
                               best.data_ptr(), _ptr(ws), need, raw))
    return LogProbs(None if tokens is None else logp, lse, entropy, ids, best if top > 0 else None)


def logprobs_backward(logits, tokens, lse, entropy, g_logp=None, g_entropy=None, out=None, stream=None):
    """Gradient of sum g_logp logp + g_entropy entropy with respect to the logits, in their type; `out` may be the logits.
    lse and entropy are those of `logprobs`; see lsam_logprobs_backward."""
    L = _ready or _lib()
    d = _logprobs_desc(logits, 0)
    rows = logits.shape[0]
    if tokens is not None:
        _expect(tokens, "tokens", logits, (rows,), torch.int32, True)
    _expect(lse, "lse", logits, (rows, 2), torch.float32, True)
    for t, what in ((entropy, "the entropy"), (g_logp, "g_logp"), (g_entropy, "g_entropy")):
        if t is not None:
            _expect(t, what, logits, (rows,), torch.float32, True)
    if out is not None:
        _expect(out, "out", logits, logits.shape, logits.dtype)
    with _On(logits, stream) as raw:
        dz = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device) if out is None else out
        _check(L.lsam_logprobs_backward(C.byref(d), logits.data_ptr(), _ptr(tokens), lse.data_ptr(), _ptr(entropy),
                                        _ptr(g_logp), _ptr(g_entropy), dz.data_ptr(), dz.stride(0), raw))
    return dz


Recurrence = namedtuple("Recurrence", "h last states")


def _recurrence_desc(f, x, h0, offsets):
    n = 3 if offsets is None else 2
    if f.dim() != n:
        _refuse("f has %d indices: [seqs, rows, dim] is wanted, or [rows, dim] with offsets" % f.dim())
    _expect(f, "f")
    _expect(x, "x", f, f.shape, f.dtype)
    if offsets is None:
        seqs, rows, dim = f.shape
    else:
        if offsets.dim() != 1 or offsets.shape[0] < 1:
            _refuse("the offsets must be [seqs + 1]")
        _expect(offsets, "the offsets", f, None, torch.int64, True)
        seqs, (rows, dim) = offsets.shape[0] - 1, f.shape
    if h0 is not None:
        _expect(h0, "h0", f, (seqs, dim), torch.float32, True)
    return lsam_recurrence_desc(seqs, rows, dim, _dtype(f, "f"), n == 2, _rows(f), _rows(x))


def _rows(t):
    s = t.stride()
    return (s[0], 0) if len(s) == 2 else (s[1], s[0])


def recurrence(f, x, h0=None, offsets=None, save=False, out=None, stream=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(f), along sequences of equal length (f, x: [seqs, rows, dim]) or
    packed ones (f, x: [rows, dim], offsets: int64 [seqs + 1]); see lsam_recurrence.  Returns h in x's type, the last
    states [seqs, dim] in fp32, and with `save` the states that `recurrence_backward` takes (else None).  Rows of no
    sequence are not written."""
    L = _ready or _lib()
    d = _recurrence_desc(f, x, h0, offsets)
    if out is not None:
        _expect(out, "out", f, f.shape, f.dtype)
    at, device = C.byref(d), f.device
    with _On(f, stream) as raw:
        h = torch.empty(f.shape, dtype=f.dtype, device=device) if out is None else out
        d.h = _rows(h)
        last = torch.empty((d.seqs, d.dim), dtype=torch.float32, device=device)
        states = torch.empty((_check(L.lsam_recurrence_states(at)), d.dim), dtype=torch.float32, device=device) if save else None
        need = L.lsam_recurrence_workspace_bytes(at)
        ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        _check(L.lsam_recurrence(at, _ptr(offsets), f.data_ptr(), x.data_ptr(), _ptr(h0), h.data_ptr(), last.data_ptr(), _ptr(states),
                                 _ptr(ws), need, raw))
    return Recurrence(h, last, states)


def recurrence_backward(f, x, dh, states, h0=None, dlast=None, offsets=None, df=None, dx=None, stream=None):
    """Gradients (df, dx, dh0) of sum dh h + dlast last; `states` are those that `recurrence` saved for the same f, x, h0 and
    offsets.  df and dx have x's type, dh0 is fp32.  Rows of no sequence are not written."""
    L = _ready or _lib()
    d = _recurrence_desc(f, x, h0, offsets)
    _expect(dh, "dh", f, f.shape, f.dtype)
    if dlast is not None:
        _expect(dlast, "dlast", f, (d.seqs, d.dim), torch.float32, True)
    for t, what in ((df, "df"), (dx, "dx")):
        if t is not None:
            _expect(t, what, f, f.shape, f.dtype)
    at, device = C.byref(d), f.device
    _expect(states, "the states", f, (_check(L.lsam_recurrence_states(at)), d.dim), torch.float32, True)
    with _On(f, stream) as raw:
        df = torch.empty(f.shape, dtype=f.dtype, device=device) if df is None else df
        dx = torch.empty(f.shape, dtype=f.dtype, device=device) if dx is None else dx
        dh0 = torch.empty((d.seqs, d.dim), dtype=torch.float32, device=device)
        d.dh, d.df, d.dx = _rows(dh), _rows(df), _rows(dx)
        need = L.lsam_recurrence_workspace_bytes(at)
        ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        _check(L.lsam_recurrence_backward(at, _ptr(offsets), f.data_ptr(), x.data_ptr(), _ptr(h0), states.data_ptr(), dh.data_ptr(),
                                          _ptr(dlast), df.data_ptr(), dx.data_ptr(), dh0.data_ptr(), _ptr(ws), need, raw))
    return df, dx, dh0


def _adapter_desc(x, W, A, B, seg_begin, seg_adapter, scale):
    for t, what, n in ((x, "x", 2), (W, "W", 2), (A, "A", 3), (B, "B", 3)):
        if t.dim() != n:
            _refuse("%s has %d indices: %d are wanted" % (what, t.dim(), n))
    _expect(x, "x")
    (rows, inp), out, (adapters, rank, _) = x.shape, W.shape[0], A.shape
    _expect(W, "W", x, (out, inp), x.dtype)
    _expect(A, "A", x, (adapters, rank, inp))
    _expect(B, "B", x, (adapters, out, rank), A.dtype)
    _expect(seg_adapter, "seg_adapter", x, None, torch.int32, True)
    segs = seg_adapter.numel()
    _expect(seg_begin, "seg_begin", x, (segs + 1,), torch.int32, True)
    a, b = A.stride(), B.stride()
    return lsam_adapter_desc(rows, inp, out, rank, adapters, segs, _dtype(x, "x"), _dtype(A, "A"), scale, x.stride(0), W.stride(0), 0,
                             a[0], a[1], b[0], b[1])


def adapter(x, W, A, B, seg_begin, seg_adapter, scale, bias=None, out=None, stream=None):
    """x W^T + bias + scale (x A_a^T) B_a^T for x [rows, in], W [out, in], A [adapters, rank, in], B [adapters, out, rank], a the adapter of
    the row's segment (seg_begin: int32 [segs + 1], seg_adapter: int32 [segs]; -1: none); see lsam_adapter.  Returns the
    result in x's type and u = x A_a^T [rows, rank] in fp32, which `adapter_backward` takes.  A and B may be parts of one
    [adapters, d] array."""
    L = _ready or _lib()
    d = _adapter_desc(x, W, A, B, seg_begin, seg_adapter, scale)
    if bias is not None:
        _expect(bias, "the bias", x, (d.out,), torch.float32, True)
    if out is not None:
        _expect(out, "out", x, (d.rows, d.out), x.dtype)
    with _On(x, stream) as raw:
        y = torch.empty((d.rows, d.out), dtype=x.dtype, device=x.device) if out is None else out
        u = torch.empty((d.rows, d.rank), dtype=torch.float32, device=x.device)
        d.y_stride = y.stride(0)
        need = L.lsam_adapter_workspace_bytes(C.byref(d), 0)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        _check(L.lsam_adapter(C.byref(d), x.data_ptr(), W.data_ptr(), _ptr(bias), A.data_ptr(), B.data_ptr(), seg_begin.data_ptr(),
                              seg_adapter.data_ptr(), u.data_ptr(), y.data_ptr(), _ptr(ws), need, raw))
    return y, u


def adapter_backward(x, W, A, B, u, dy, seg_begin, seg_adapter, scale, dx=None, dA=None, dB=None, want_dx=True, want_adapters=True,
                     stream=None):
    """Gradients (dx, dA, dB) of `adapter` for dy [rows, out]: dx in x's type, dA and dB in fp32, written whole.  dA and dB may be
    parts of one [adapters, d] array, as gradients that go to lsam_step_grads are.  What is not wanted is None."""
    L = _ready or _lib()
    d = _adapter_desc(x, W, A, B, seg_begin, seg_adapter, scale)
    _expect(dy, "dy", x, (d.rows, d.out), x.dtype)
    _expect(u, "u", x, (d.rows, d.rank), torch.float32, True)
    for t, what, shape, dtype in ((dx, "dx", x.shape, x.dtype), (dA, "dA", A.shape, torch.float32), (dB, "dB", B.shape, torch.float32)):
        if t is not None:
            _expect(t, what, x, shape, dtype)
    with _On(x, stream) as raw:
        new = lambda like, dtype: torch.empty(like.shape, dtype=dtype, device=x.device)  # noqa: E731
        dx = (new(x, x.dtype) if dx is None else dx) if want_dx else None
        dA = (new(A, torch.float32) if dA is None else dA) if want_adapters else None
        dB = (new(B, torch.float32) if dB is None else dB) if want_adapters else None
        d.dy_stride = dy.stride(0)
        if want_dx:
            d.dx_stride = dx.stride(0)
        if want_adapters:
            d.da_adapter, d.da_stride = dA.stride()[:2]
            d.db_adapter, d.db_stride = dB.stride()[:2]
        need = L.lsam_adapter_workspace_bytes(C.byref(d), 1)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        _check(L.lsam_adapter_backward(C.byref(d), x.data_ptr(), W.data_ptr(), A.data_ptr(), B.data_ptr(), seg_begin.data_ptr(),
                                       seg_adapter.data_ptr(), u.data_ptr(), dy.data_ptr(), _ptr(dx), _ptr(dA), _ptr(dB), _ptr(ws),
                                       need, raw))
    return dx, dA, dB
