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
EMBEDDING_MAX_VOCAB = 1 << 22
RESIDUAL_MAX_DIM = 16384
ATTENTION_MAX_DIM = 128

EXPORTS = ["lsam_dropout", "lsam_logprobs_workspace_bytes", "lsam_logprobs", "lsam_logprobs_backward",
           "lsam_recurrence_workspace_bytes", "lsam_recurrence_states", "lsam_recurrence", "lsam_recurrence_backward",
           "lsam_adapter_workspace_bytes", "lsam_adapter", "lsam_adapter_backward",
           "lsam_embedding", "lsam_embedding_workspace_bytes", "lsam_embedding_backward",
           "lsam_residual", "lsam_residual_workspace_bytes", "lsam_residual_backward",
           "lsam_attention", "lsam_attention_workspace_bytes", "lsam_attention_backward",
           "lsam_attention_step_workspace_bytes", "lsam_attention_step"]


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


class lsam_embedding_desc(C.Structure):
    _fields_ = [("replicas", C.c_int32), ("dtype", C.c_int32), ("table_dtype", C.c_int32), ("scale", C.c_float)] + [
        (n, C.c_int64) for n in ("rows", "vocab", "dim", "token_replica", "table_stride", "table_replica", "y_stride", "y_replica",
                                 "dy_stride", "dy_replica", "dtable_stride", "dtable_replica")]


class lsam_residual_desc(C.Structure):
    _fields_ = [("replicas", C.c_int32), ("dtype", C.c_int32), ("rows", C.c_int64), ("dim", C.c_int64), ("alpha", C.c_float),
                ("beta", C.c_float), ("eps", C.c_float)] + [
                    (n, C.c_int64) for n in ("w_pre_replica", "w_post_replica", "r_stride", "r_replica", "y_stride", "y_replica",
                                             "gate_stride", "gate_replica", "r_out_stride", "r_out_replica", "h_stride", "h_replica",
                                             "dr_stride", "dr_replica", "dh_stride", "dh_replica", "dr_out_stride", "dr_out_replica",
                                             "dy_stride", "dy_replica", "dgate_stride", "dgate_replica", "dw_pre_replica",
                                             "dw_post_replica")]


class lsam_heads(C.Structure):
    _fields_ = [("stride", C.c_int64), ("head", C.c_int64)]


class lsam_attention_desc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("seqs", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32), ("dtype", C.c_int32),
                ("scale", C.c_float)] + [(n, lsam_heads) for n in ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")]


class lsam_attention_step_desc(C.Structure):
    _fields_ = [("seqs", C.c_int64), ("capacity", C.c_int64), ("prefix", C.c_int64), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("dim", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float), ("q", lsam_heads), ("o", lsam_heads), ("k", lsam_heads),
                ("v", lsam_heads), ("k_seq", C.c_int64), ("v_seq", C.c_int64), ("prefix_k", lsam_heads), ("prefix_v", lsam_heads)]


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
        emb, res = C.POINTER(lsam_embedding_desc), C.POINTER(lsam_residual_desc)
        L.lsam_embedding.restype = C.c_int
        L.lsam_embedding.argtypes = [emb] + [vp] * 4
        L.lsam_embedding_workspace_bytes.restype = C.c_size_t
        L.lsam_embedding_workspace_bytes.argtypes = [emb]
        L.lsam_embedding_backward.restype = C.c_int
        L.lsam_embedding_backward.argtypes = [emb] + [vp] * 4 + [C.c_size_t, vp]
        L.lsam_residual.restype = C.c_int
        L.lsam_residual.argtypes = [res] + [vp] * 8
        L.lsam_residual_workspace_bytes.restype = C.c_size_t
        L.lsam_residual_workspace_bytes.argtypes = [res]
        L.lsam_residual_backward.restype = C.c_int
        L.lsam_residual_backward.argtypes = [res] + [vp] * 13 + [C.c_size_t, vp]
        att = C.POINTER(lsam_attention_desc)
        L.lsam_attention.restype = C.c_int
        L.lsam_attention.argtypes = [att] + [vp] * 7
        L.lsam_attention_workspace_bytes.restype = C.c_size_t
        L.lsam_attention_workspace_bytes.argtypes = [att]
        L.lsam_attention_backward.restype = C.c_int
        L.lsam_attention_backward.argtypes = [att] + [vp] * 11 + [C.c_size_t, vp]
        step = C.POINTER(lsam_attention_step_desc)
        L.lsam_attention_step_workspace_bytes.restype = C.c_size_t
        L.lsam_attention_step_workspace_bytes.argtypes = [step]
        L.lsam_attention_step.restype = C.c_int
        L.lsam_attention_step.argtypes = [step] + [vp] * 8 + [C.c_size_t, vp]
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


def _of_replicas(t):
    """Strides from row to row and from replica to replica; without the latter index there is one replica."""
    s = t.stride()
    return (s[0], 0) if len(s) == 2 else (s[1], s[0])


def _embedding_tokens(tokens):
    if not 1 <= tokens.dim() <= 2:
        _refuse("the tokens have %d indices: [rows] or [K, rows] is wanted" % tokens.dim())
    _expect(tokens, "the tokens", None, None, torch.int32)
    return (1, tokens.shape[0], 0) if tokens.dim() == 1 else (tokens.shape[0], tokens.shape[1], tokens.stride(0))


def embedding(tokens, table, scale=1.0, dtype=None, out=None, stream=None):
    """scale * table[token] in `dtype` (the table's, or out's): tokens [rows] and one table [vocab, dim], or tokens [K, rows] of K replicas and their tables
    [K, vocab, dim], or one table [vocab, dim] that all read.  A token outside the vocabulary has a row of zeros; see
    lsam_embedding."""
    L = _ready or _lib()
    K, rows, apart = _embedding_tokens(tokens)
    n = table.dim()
    if not 2 <= n <= tokens.dim() + 1:
        _refuse("the table has %d indices: [vocab, dim] is wanted, or [K, vocab, dim] for tokens [K, rows]" % n)
    _expect(table, "the table", tokens, (K,) + tuple(table.shape[1:]) if n == 3 else None)
    vocab, dim = table.shape[-2:]
    shape = tuple(tokens.shape) + (dim,)
    if out is not None:
        _expect(out, "out", tokens, shape, dtype)
    with _On(tokens, stream) as raw:
        y = torch.empty(shape, dtype=table.dtype if dtype is None else dtype, device=tokens.device) if out is None else out
        d = lsam_embedding_desc(K, _dtype(y, "the result"), _dtype(table, "the table"), scale, rows, vocab, dim, apart, *_of_replicas(table),
                                *_of_replicas(y))
        _check(L.lsam_embedding(C.byref(d), tokens.data_ptr(), table.data_ptr(), y.data_ptr(), raw))
    return y


def embedding_backward(tokens, dy, vocab, scale=1.0, out=None, stream=None):
    """Gradient of the tables in fp32, [vocab, dim] or [K, vocab, dim], written whole: scale times the sum of each token's rows of dy (tokens'
    shape + [dim]).  The gradient of a table that K replicas share is that of their tokens and dy as one replica's: tokens.view(-1).  `out` may be
    part of one [K, d] array; see lsam_embedding_backward."""
    L = _ready or _lib()
    K, rows, apart = _embedding_tokens(tokens)
    if dy.dim() != tokens.dim() + 1:
        _refuse("dy has %d indices: %d are wanted" % (dy.dim(), tokens.dim() + 1))
    _expect(dy, "dy", tokens, tuple(tokens.shape) + (dy.shape[-1],))
    shape = tuple(tokens.shape[:-1]) + (vocab, dy.shape[-1])
    if out is not None:
        _expect(out, "out", tokens, shape, torch.float32)
    d = lsam_embedding_desc(K, _dtype(dy, "dy"), DTYPE_FP32, scale, rows, vocab, dy.shape[-1], apart, 0, 0, 0, 0, *_of_replicas(dy))
    at = C.byref(d)
    with _On(tokens, stream) as raw:
        need = L.lsam_embedding_workspace_bytes(at)
        if need == 0 and K > 0:
            _refuse(lsam.last_error())
        dtable = torch.empty(shape, dtype=torch.float32, device=tokens.device) if out is None else out
        d.dtable_stride, d.dtable_replica = _of_replicas(dtable)
        ws = torch.empty(need, dtype=torch.uint8, device=tokens.device) if need else None
        _check(L.lsam_embedding_backward(at, tokens.data_ptr(), dy.data_ptr(), dtable.data_ptr(), _ptr(ws), need, raw))
    return dtable


ResidualGradients = namedtuple("ResidualGradients", "dr dy dgate dw_pre dw_post")


_NO_ROWS = (0, 0)


def _residual_desc(r, y, w_pre, w_post, gate, alpha, beta, eps, outs):
    """`outs`: strides from row to row and from replica to replica of what comes behind the gate in the descriptor."""
    n, shape = r.dim(), r.shape
    _expect(r, "r")
    if y is not None:
        _expect(y, "y", r, shape, r.dtype)
    if gate is not None:
        _expect(gate, "the gate", r, shape, r.dtype)
    K, rows, dim = shape if n == 3 else (1,) + shape
    apart = [0, 0]
    for i, (t, what) in enumerate(((w_pre, "w_pre"), (w_post, "w_post"))):
        if t is not None:
            one = t.dim() == 1
            _expect(t, what, r, (dim,) if one else (K, dim), torch.float32)
            if not one:
                apart[i] = t.stride(0)
    return lsam_residual_desc(K, _dtype(r, "r"), rows, dim, alpha, beta, eps, *apart, *_of_replicas(r), *(_NO_ROWS if y is None else _of_replicas(y)),
                              *(_NO_ROWS if gate is None else _of_replicas(gate)), *outs)


def _strides(*tensors):
    s = []
    for t in tensors:
        s += _NO_ROWS if t is None else _of_replicas(t)
    return s


def residual(r, y, w_pre, w_post=None, gate=None, alpha=1.0, beta=1.0, eps=1e-6, out=None, h=None, stream=None):
    """(r', h) with r' = alpha r + beta sigmoid(gate) w_post n(y) and h = w_pre n(r'), n(x) = x / sqrt(mean x^2 + eps): what a block made of the
    stream r joins it, and the stream as the next block reads it.  r, y, gate: [rows, dim], or [K, rows, dim] of K replicas; weights fp32 [dim],
    or [K, dim].  No gate, no w_post (y as it is), no w_pre (h is None) and no y (r' is r itself) are possible; `out` for r' may be r; see
    lsam_residual."""
    L = _ready or _lib()
    if not 2 <= r.dim() <= 3:
        _refuse("r has %d indices: [rows, dim] or [K, rows, dim] is wanted" % r.dim())
    for t, what in ((out, "out"), (h, "h")):
        if t is not None:
            _expect(t, what, r, r.shape, r.dtype)
    with _On(r, stream) as raw:
        new = None if y is None else torch.empty(r.shape, dtype=r.dtype, device=r.device) if out is None else out
        h = None if w_pre is None else torch.empty(r.shape, dtype=r.dtype, device=r.device) if h is None else h
        d = _residual_desc(r, y, w_pre, w_post, gate, alpha, beta, eps, _strides(new, h))
        _check(L.lsam_residual(C.byref(d), r.data_ptr(), _ptr(y), _ptr(gate), _ptr(w_pre), _ptr(w_post), _ptr(new), _ptr(h), raw))
    return r if y is None else new, h


def residual_backward(r, y, w_pre, dr, dh, w_post=None, gate=None, alpha=1.0, beta=1.0, eps=1e-6, dr_out=None, dy=None, dgate=None, dw_pre=None,
                      dw_post=None, want_weights=True, stream=None):
    """Gradients (dr, dy, dgate, dw_pre, dw_post) of `residual` for the gradients dr of r' (or None: 0) and dh of h; r is r' as `residual` left it.
    Those of the weights are fp32, written whole; weights of K replicas are [K, dim], and their gradients may be parts of one [K, d]
    array.  dr_out may be dr.  What has no gradient is None; see lsam_residual_backward."""
    L = _ready or _lib()
    if not 2 <= r.dim() <= 3:
        _refuse("r has %d indices: [rows, dim] or [K, rows, dim] is wanted" % r.dim())
    if y is None:
        w_post = gate = None
    for t, what in ((w_pre, "w_pre"), (w_post, "w_post")):
        if want_weights and t is not None and t.dim() != r.dim() - 1:
            _refuse("%s is shared by replicas: pass their rows as one replica's for its gradient" % what)
    for t, what in ((dr, "dr"), (dh, "dh"), (dr_out, "dr_out"), (dy, "dy"), (dgate, "dgate")):
        if t is not None:
            _expect(t, what, r, r.shape, r.dtype)
    if w_pre is not None and dh is None:
        _refuse("dh is missing: there is a w_pre")
    for t, what, w in ((dw_pre, "dw_pre", w_pre), (dw_post, "dw_post", w_post)):
        if t is not None and w is not None:
            _expect(t, what, r, w.shape, torch.float32)
    device = r.device
    with _On(r, stream) as raw:
        new = lambda t, like, dtype: torch.empty(like.shape, dtype=dtype, device=device) if t is None else t  # noqa: E731
        dr_out = new(dr_out, r, r.dtype)
        dy = new(dy, r, r.dtype) if y is not None else None
        dgate = new(dgate, r, r.dtype) if gate is not None else None
        dw_pre = new(dw_pre, w_pre, torch.float32) if want_weights and w_pre is not None else None
        dw_post = new(dw_post, w_post, torch.float32) if want_weights and w_post is not None else None
        apart = [0 if t is None or t.dim() == 1 else t.stride(0) for t in (dw_pre, dw_post)]
        d = _residual_desc(r, y, w_pre, w_post, gate, alpha, beta, eps, _strides(None, None, dr, dh, dr_out, dy, dgate) + apart)
        at = C.byref(d)
        need = L.lsam_residual_workspace_bytes(at) if dw_pre is not None or dw_post is not None else 0
        ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        _check(L.lsam_residual_backward(at, r.data_ptr(), _ptr(y), _ptr(gate), _ptr(w_pre), _ptr(w_post), _ptr(dr), _ptr(dh), dr_out.data_ptr(),
                                        _ptr(dy), _ptr(dgate), _ptr(dw_pre), _ptr(dw_post), _ptr(ws), need, raw))
    return ResidualGradients(dr_out, dy, dgate, dw_pre, dw_post)


Attention = namedtuple("Attention", "o lse")


def _scale(dim, scale):
    return max(dim, 1) ** -0.5 if scale is None else scale


def _attention_desc(q, k, v, offsets, scale):
    for t, what in ((q, "q"), (k, "k"), (v, "v")):
        if t.dim() != 3:
            _refuse("%s has %d indices: [rows, heads, dim] is wanted" % (what, t.dim()))
    if offsets.dim() != 1 or offsets.shape[0] < 1:
        _refuse("the offsets must be [seqs + 1]")
    _expect(q, "q")
    rows, heads, dim = q.shape
    kv_heads = k.shape[1]
    _expect(k, "k", q, (rows, kv_heads, dim), q.dtype)
    _expect(v, "v", q, (rows, kv_heads, dim), q.dtype)
    _expect(offsets, "the offsets", q, None, torch.int64, True)
    return lsam_attention_desc(rows, offsets.shape[0] - 1, heads, kv_heads, dim, _dtype(q, "q"), _scale(dim, scale),
                               q.stride()[:2], k.stride()[:2], v.stride()[:2])


def attention(q, k, v, offsets, scale=None, save=False, out=None, stream=None):
    """Causal attention of packed sequences: o [rows, heads, dim] = softmax(scale q k) v for q [rows, heads, dim] and k, v [rows, kv_heads, dim],
    heads a multiple of kv_heads, sequence s the rows offsets[s] .. offsets[s + 1] - 1 (int64 [seqs + 1]); scale is dim^-0.5 where none is
    given.  Returns (o, lse), lse [heads, rows] in fp32 with `save`, for `attention_backward`, else None.  Rows of no sequence are not written;
    see lsam_attention."""
    L = _ready or _lib()
    d = _attention_desc(q, k, v, offsets, scale)
    if out is not None:
        _expect(out, "out", q, q.shape, q.dtype)
    with _On(q, stream) as raw:
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        d.o = o.stride()[:2]
        lse = torch.empty((d.heads, d.rows), dtype=torch.float32, device=q.device) if save else None
        _check(L.lsam_attention(C.byref(d), offsets.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _ptr(lse), raw))
    return Attention(o, lse)


def attention_backward(q, k, v, offsets, o, lse, do, scale=None, dq=None, dk=None, dv=None, stream=None):
    """Gradients (dq, dk, dv) of `attention` for the gradient do of o, in their types; o and lse are those it returned.  Rows of no sequence are not
    written; see lsam_attention_backward."""
    L = _ready or _lib()
    d = _attention_desc(q, k, v, offsets, scale)
    for t, what in ((o, "o"), (do, "do"), (dq, "dq")):
        if t is not None:
            _expect(t, what, q, q.shape, q.dtype)
    for t, what in ((dk, "dk"), (dv, "dv")):
        if t is not None:
            _expect(t, what, q, k.shape, q.dtype)
    _expect(lse, "lse", q, (d.heads, d.rows), torch.float32, True)
    at, device = C.byref(d), q.device
    with _On(q, stream) as raw:
        dq = torch.empty(q.shape, dtype=q.dtype, device=device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=q.dtype, device=device) if dk is None else dk
        dv = torch.empty(k.shape, dtype=q.dtype, device=device) if dv is None else dv
        d.o, d.d_o, d.dq, d.dk, d.dv = (t.stride()[:2] for t in (o, do, dq, dk, dv))
        need = L.lsam_attention_workspace_bytes(at)
        ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        _check(L.lsam_attention_backward(at, offsets.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), do.data_ptr(),
                                         dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(ws), need, raw))
    return dq, dk, dv


def attention_step(q, k, v, lengths, prefix_k=None, prefix_v=None, scale=None, out=None, stream=None):
    """One token of each sequence: softmax(scale q k) v [seqs, heads, dim] over the prefix [prefix, kv_heads, dim], which all sequences share, and
    the first lengths[s] (int32 [seqs]) places of the caches k, v [seqs, capacity, kv_heads, dim]; 0 where both are empty.  scale is dim^-0.5 where
    none is given; see lsam_attention_step."""
    L = _ready or _lib()
    for t, what, n in ((q, "q", 3), (k, "k", 4), (v, "v", 4), (prefix_k, "prefix_k", 3), (prefix_v, "prefix_v", 3)):
        if t is not None and t.dim() != n:
            _refuse("%s has %d indices: %d are wanted" % (what, t.dim(), n))
    if (prefix_k is None) != (prefix_v is None):
        _refuse("of prefix_k and prefix_v one is missing")
    _expect(q, "q")
    (seqs, heads, dim), (_, capacity, kv_heads, _) = q.shape, k.shape
    _expect(k, "k", q, (seqs, capacity, kv_heads, dim), q.dtype)
    _expect(v, "v", q, (seqs, capacity, kv_heads, dim), q.dtype)
    _expect(lengths, "the lengths", q, (seqs,), torch.int32, True)
    prefix, pk, pv = 0, (0, 0), (0, 0)
    if prefix_k is not None:
        prefix = prefix_k.shape[0]
        _expect(prefix_k, "prefix_k", q, (prefix, kv_heads, dim), q.dtype)
        _expect(prefix_v, "prefix_v", q, (prefix, kv_heads, dim), q.dtype)
        pk, pv = prefix_k.stride()[:2], prefix_v.stride()[:2]
    if out is not None:
        _expect(out, "out", q, q.shape, q.dtype)
    ks, vs = k.stride(), v.stride()
    with _On(q, stream) as raw:
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        d = lsam_attention_step_desc(seqs, capacity, prefix, heads, kv_heads, dim, _dtype(q, "q"), _scale(dim, scale),
                                     q.stride()[:2], o.stride()[:2], ks[1:3], vs[1:3], ks[0], vs[0], pk, pv)
        need = L.lsam_attention_step_workspace_bytes(C.byref(d))
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        _check(L.lsam_attention_step(C.byref(d), lengths.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(prefix_k), _ptr(prefix_v),
                                     o.data_ptr(), _ptr(ws), need, raw))
    return o
