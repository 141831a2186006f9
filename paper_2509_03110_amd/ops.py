"""ctypes binding of the operators in include/lsam_ops.h: argument marshalling only.

Tensors are checked for what the C boundary cannot see (device, type, shape, contiguous last index) and handed over
as they lie, strides included.  Outputs that are not given are allocated on the stream that the call runs on: the
current stream of x's device, or `stream` (a torch.cuda.Stream).  As with any torch operation, inputs that were made
on another stream have to be ready on this one, and tensors that are dropped while another stream still reads them
need record_stream.  Gradients are entry points of their own; nothing here records for autograd.
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


def _lib():
    global _ready
    if _ready is None:
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


_types = None


def _dtype(t, what):
    global _types
    if _types is None:
        import torch
        _types = {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16}
    code = _types.get(t.dtype)
    if code is None:
        _refuse("%s is %s: float32 or bfloat16 is wanted" % (what, t.dtype))
    return code


def _expect(t, what, like=None, shape=None, dtype=None, dense=False):
    """Whether `t` is a tensor of that device, shape and type with a contiguous last index (dense: all of it)."""
    if like is not None and t.device != like.device:
        _refuse("%s is on %s, not on %s" % (what, t.device, like.device))
    if not t.is_cuda:
        _refuse("%s is not on a GPU" % what)
    if shape is not None and tuple(t.shape) != tuple(shape):
        _refuse("%s has shape %s: %s is wanted" % (what, tuple(t.shape), tuple(shape)))
    if dtype is not None and t.dtype != dtype:
        _refuse("%s is %s: %s is wanted" % (what, t.dtype, dtype))
    if dense:
        if not t.is_contiguous():
            _refuse("%s must be contiguous" % what)
    elif t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("the last index of %s must be contiguous" % what)


class _On:
    """The device and stream that a call runs on, current while it lasts; `.raw` is the stream's handle."""

    def __init__(self, t, stream):
        import torch
        self.device, self.context = t.device, None
        if stream is not None:
            if stream.device != t.device:
                _refuse("the stream belongs to %s, the tensors to %s" % (stream.device, t.device))
            self.context = torch.cuda.stream(stream)
        elif torch.cuda.current_device() != t.device.index:
            self.context = torch.cuda.device(t.device)

    def __enter__(self):
        import torch
        if self.context is not None:
            self.context.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *err):
        if self.context is not None:
            self.context.__exit__(*err)


def _ptr(t):
    return None if t is None else t.data_ptr()


def dropout(x, p, seed, step, site=0, first_replica=0, residual=None, out=None, stream=None):
    """residual + m x / (1 - p) with the mask m of (seed, step, site, place); see lsam_dropout.  x: [K, rows, cols]
    of K replicas, [rows, cols] or [cols] of one.  The gradient of x is the same call on the gradient of the result,
    with no residual.  `out` may be x or the residual."""
    import torch
    if not 1 <= x.dim() <= 3:
        _refuse("x has %d indices: 1 to 3 are wanted" % x.dim())
    _expect(x, "x")
    for t, what in ((residual, "the residual"), (out, "out")):
        if t is not None:
            _expect(t, what, like=x, shape=x.shape, dtype=x.dtype)
    d = lsam_dropout_desc()
    d.dtype = _dtype(x, "x")
    shape = (1,) * (3 - x.dim()) + tuple(x.shape)
    d.replicas, d.rows, d.cols = shape
    if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 32 and 0 <= site < 1 << 16 and 0 <= first_replica < 1 << 16):
        _refuse("the seed has 64 bits, the step 32, the site and the replica 16")
    d.p, d.seed, d.step, d.site, d.first_replica = p, seed, step, site, first_replica

    def strides(t):
        return (0,) * (2 - t.dim() + 1) + tuple(t.stride()) if t.dim() < 3 else t.stride()
    with _On(x, stream) as raw:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        d.x_replica, d.x_stride = strides(x)[:2]
        d.y_replica, d.y_stride = strides(y)[:2]
        if residual is not None:
            d.residual_replica, d.residual_stride = strides(residual)[:2]
        _check(_lib().lsam_dropout(C.byref(d), x.data_ptr(), _ptr(residual), y.data_ptr(), raw))
    return y


LogProbs = namedtuple("LogProbs", "logp lse entropy top_ids top_logp")


def _logprobs_desc(logits, top):
    if logits.dim() != 2:
        _refuse("the logits have %d indices: [rows, vocab] is wanted" % logits.dim())
    _expect(logits, "logits")
    d = lsam_logprobs_desc()
    d.rows, d.vocab = logits.shape
    d.stride, d.dtype, d.top = logits.stride(0), _dtype(logits, "logits"), top
    return d


def logprobs(logits, tokens=None, top=0, stream=None):
    """Log probabilities of tokens [rows] (int32; one outside the vocabulary does not count: 0) under logits
    [rows, vocab], with the log normaliser in two parts lse [rows, 2] (the largest logit m, and ln sum e^{z - m}), the
    entropy [rows], and the `top` largest logits' indices and log probabilities [rows, top]; see lsam_logprobs.  Fields that were not asked for
    are None."""
    import torch
    d = _logprobs_desc(logits, top)
    if tokens is not None:
        _expect(tokens, "tokens", like=logits, shape=(d.rows,), dtype=torch.int32, dense=True)
    with _On(logits, stream) as raw:
        new = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device=logits.device)  # noqa: E731
        need = _lib().lsam_logprobs_workspace_bytes(C.byref(d))
        ws = new(need, t=torch.uint8) if need else None
        r = LogProbs(None if tokens is None else new(d.rows), new(d.rows, 2), new(d.rows),
                     new(d.rows, top, t=torch.int32) if top > 0 else None, new(d.rows, top) if top > 0 else None)
        _check(_lib().lsam_logprobs(C.byref(d), logits.data_ptr(), _ptr(tokens), _ptr(r.logp), r.lse.data_ptr(),
                                    r.entropy.data_ptr(), _ptr(r.top_ids), _ptr(r.top_logp), _ptr(ws), need, raw))
    return r


def logprobs_backward(logits, tokens, lse, entropy, g_logp=None, g_entropy=None, out=None, stream=None):
    """Gradient of sum g_logp logp + g_entropy entropy with respect to the logits, in their type; `out` may be the logits.
    lse and entropy are those of `logprobs`; see lsam_logprobs_backward."""
    import torch
    d = _logprobs_desc(logits, 0)
    if tokens is not None:
        _expect(tokens, "tokens", like=logits, shape=(d.rows,), dtype=torch.int32, dense=True)
    _expect(lse, "lse", like=logits, shape=(d.rows, 2), dtype=torch.float32, dense=True)
    for t, what in ((entropy, "the entropy"), (g_logp, "g_logp"), (g_entropy, "g_entropy")):
        if t is not None:
            _expect(t, what, like=logits, shape=(d.rows,), dtype=torch.float32, dense=True)
    if out is not None:
        _expect(out, "out", like=logits, shape=logits.shape, dtype=logits.dtype)
    with _On(logits, stream) as raw:
        dz = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device) if out is None else out
        _check(_lib().lsam_logprobs_backward(C.byref(d), logits.data_ptr(), _ptr(tokens), lse.data_ptr(), _ptr(entropy),
                                             _ptr(g_logp), _ptr(g_entropy), dz.data_ptr(), dz.stride(0), raw))
    return dz


Recurrence = namedtuple("Recurrence", "h last states")


def _recurrence_desc(f, x, h0, offsets):
    import torch
    if f.dim() != (3 if offsets is None else 2):
        _refuse("f has %d indices: [seqs, rows, dim] is wanted, or [rows, dim] with offsets" % f.dim())
    _expect(f, "f")
    _expect(x, "x", like=f, shape=f.shape, dtype=f.dtype)
    d = lsam_recurrence_desc()
    d.dtype = _dtype(f, "f")
    if offsets is None:
        d.seqs, d.rows, d.dim = f.shape
    else:
        if offsets.dim() != 1 or offsets.shape[0] < 1:
            _refuse("the offsets must be [seqs + 1]")
        _expect(offsets, "the offsets", like=f, dtype=torch.int64, dense=True)
        d.packed, d.seqs, (d.rows, d.dim) = 1, offsets.shape[0] - 1, f.shape
    if h0 is not None:
        _expect(h0, "h0", like=f, shape=(d.seqs, d.dim), dtype=torch.float32, dense=True)
    _rows(d.f, f)
    _rows(d.x, x)
    return d


def _rows(at, t):
    at.seq, at.stride = (0, t.stride(0)) if t.dim() == 2 else t.stride()[:2]


def recurrence(f, x, h0=None, offsets=None, save=False, out=None, stream=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(f), along sequences of equal length (f, x: [seqs, rows, dim]) or
    packed ones (f, x: [rows, dim], offsets: int64 [seqs + 1]); see lsam_recurrence.  Returns h in x's type, the last
    states [seqs, dim] in fp32, and with `save` the states that `recurrence_backward` takes (else None).  Rows of no
    sequence are not written."""
    import torch
    d = _recurrence_desc(f, x, h0, offsets)
    if out is not None:
        _expect(out, "out", like=f, shape=f.shape, dtype=f.dtype)
    with _On(f, stream) as raw:
        new = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device=f.device)  # noqa: E731
        h = new(*f.shape, t=f.dtype) if out is None else out
        _rows(d.h, h)
        last = new(d.seqs, d.dim)
        states = new(_check(_lib().lsam_recurrence_states(C.byref(d))), d.dim) if save else None
        need = _lib().lsam_recurrence_workspace_bytes(C.byref(d))
        ws = new(need, t=torch.uint8) if need else None
        _check(_lib().lsam_recurrence(C.byref(d), _ptr(offsets), f.data_ptr(), x.data_ptr(), _ptr(h0), h.data_ptr(),
                                      last.data_ptr(), _ptr(states), _ptr(ws), need, raw))
    return Recurrence(h, last, states)


def recurrence_backward(f, x, dh, states, h0=None, dlast=None, offsets=None, df=None, dx=None, stream=None):
    """Gradients (df, dx, dh0) of sum dh h + dlast last; `states` are those that `recurrence` saved for the same f, x, h0 and
    offsets.  df and dx have x's type, dh0 is fp32.  Rows of no sequence are not written."""
    import torch
    d = _recurrence_desc(f, x, h0, offsets)
    _expect(dh, "dh", like=f, shape=f.shape, dtype=f.dtype)
    if dlast is not None:
        _expect(dlast, "dlast", like=f, shape=(d.seqs, d.dim), dtype=torch.float32, dense=True)
    for t, what in ((df, "df"), (dx, "dx")):
        if t is not None:
            _expect(t, what, like=f, shape=f.shape, dtype=f.dtype)
    _expect(states, "the states", like=f, shape=(_check(_lib().lsam_recurrence_states(C.byref(d))), d.dim), dtype=torch.float32,
            dense=True)
    with _On(f, stream) as raw:
        new = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device=f.device)  # noqa: E731
        df = new(*f.shape, t=f.dtype) if df is None else df
        dx = new(*f.shape, t=f.dtype) if dx is None else dx
        dh0 = new(d.seqs, d.dim)
        _rows(d.dh, dh)
        _rows(d.df, df)
        _rows(d.dx, dx)
        need = _lib().lsam_recurrence_workspace_bytes(C.byref(d))
        ws = new(need, t=torch.uint8) if need else None
        _check(_lib().lsam_recurrence_backward(C.byref(d), _ptr(offsets), f.data_ptr(), x.data_ptr(), _ptr(h0), states.data_ptr(),
                                               dh.data_ptr(), _ptr(dlast), df.data_ptr(), dx.data_ptr(), dh0.data_ptr(), _ptr(ws),
                                               need, raw))
    return df, dx, dh0


def _adapter_desc(x, W, A, B, seg_begin, seg_adapter, scale):
    import torch
    for t, what, n in ((x, "x", 2), (W, "W", 2), (A, "A", 3), (B, "B", 3)):
        if t.dim() != n:
            _refuse("%s has %d indices: %d are wanted" % (what, t.dim(), n))
    _expect(x, "x")
    d = lsam_adapter_desc()
    d.rows, d.in_ = x.shape
    d.out, (d.adapters, d.rank) = W.shape[0], A.shape[:2]
    _expect(W, "W", like=x, shape=(d.out, d.in_), dtype=x.dtype)
    _expect(A, "A", like=x, shape=(d.adapters, d.rank, d.in_))
    _expect(B, "B", like=x, shape=(d.adapters, d.out, d.rank), dtype=A.dtype)
    _expect(seg_adapter, "seg_adapter", like=x, dtype=torch.int32, dense=True)
    d.segs = seg_adapter.numel()
    _expect(seg_begin, "seg_begin", like=x, shape=(d.segs + 1,), dtype=torch.int32, dense=True)
    d.dtype, d.adapter_dtype, d.scale = _dtype(x, "x"), _dtype(A, "A"), scale
    d.x_stride, d.w_stride = x.stride(0), W.stride(0)
    d.a_adapter, d.a_stride = A.stride()[:2]
    d.b_adapter, d.b_stride = B.stride()[:2]
    return d


def adapter(x, W, A, B, seg_begin, seg_adapter, scale, bias=None, out=None, stream=None):
    """x W^T + bias + scale (x A_a^T) B_a^T for x [rows, in], W [out, in], A [adapters, rank, in], B [adapters, out, rank], a the adapter of
    the row's segment (seg_begin: int32 [segs + 1], seg_adapter: int32 [segs]; -1: none); see lsam_adapter.  Returns the
    result in x's type and u = x A_a^T [rows, rank] in fp32, which `adapter_backward` takes.  A and B may be parts of one
    [adapters, d] array."""
    import torch
    d = _adapter_desc(x, W, A, B, seg_begin, seg_adapter, scale)
    if bias is not None:
        _expect(bias, "the bias", like=x, shape=(d.out,), dtype=torch.float32, dense=True)
    if out is not None:
        _expect(out, "out", like=x, shape=(d.rows, d.out), dtype=x.dtype)
    with _On(x, stream) as raw:
        y = torch.empty((d.rows, d.out), dtype=x.dtype, device=x.device) if out is None else out
        u = torch.empty((d.rows, d.rank), dtype=torch.float32, device=x.device)
        d.y_stride = y.stride(0)
        need = _lib().lsam_adapter_workspace_bytes(C.byref(d), 0)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        _check(_lib().lsam_adapter(C.byref(d), x.data_ptr(), W.data_ptr(), _ptr(bias), A.data_ptr(), B.data_ptr(), seg_begin.data_ptr(),
                                   seg_adapter.data_ptr(), u.data_ptr(), y.data_ptr(), _ptr(ws), need, raw))
    return y, u


def adapter_backward(x, W, A, B, u, dy, seg_begin, seg_adapter, scale, dx=None, dA=None, dB=None, want_dx=True, want_adapters=True,
                     stream=None):
    """Gradients (dx, dA, dB) of `adapter` for dy [rows, out]: dx in x's type, dA and dB in fp32, written whole.  dA and dB may be
    parts of one [adapters, d] array, as gradients that go to lsam_step_grads are.  What is not wanted is None."""
    import torch
    d = _adapter_desc(x, W, A, B, seg_begin, seg_adapter, scale)
    _expect(dy, "dy", like=x, shape=(d.rows, d.out), dtype=x.dtype)
    _expect(u, "u", like=x, shape=(d.rows, d.rank), dtype=torch.float32, dense=True)
    for t, what, shape, dtype in ((dx, "dx", x.shape, x.dtype), (dA, "dA", A.shape, torch.float32), (dB, "dB", B.shape, torch.float32)):
        if t is not None:
            _expect(t, what, like=x, shape=shape, dtype=dtype)
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
        need = _lib().lsam_adapter_workspace_bytes(C.byref(d), 1)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        _check(_lib().lsam_adapter_backward(C.byref(d), x.data_ptr(), W.data_ptr(), A.data_ptr(), B.data_ptr(), seg_begin.data_ptr(),
                                            seg_adapter.data_ptr(), u.data_ptr(), dy.data_ptr(), _ptr(dx), _ptr(dA), _ptr(dB), _ptr(ws),
                                            need, raw))
    return dx, dA, dB
