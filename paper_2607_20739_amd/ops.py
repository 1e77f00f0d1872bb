"""Operators that turn a language model's outputs into a partition's loss and gradient.

Binding of include/pgc_ops.h, which states what each operator computes: dropout with a mask
that is a function of seed, row number and column; log-probabilities of given tokens; the
preference loss of pairs of sequences; the clipped policy loss with a KL term.  The losses take
logits and return the loss and the logits' gradient; `logits.backward(dlogits)` carries it on
through a model.  dropout and token_logprobs take part in autograd where an input asks for it.

Tensors live on one GPU; matrices are 2-D float32, bfloat16 or float16 with adjacent columns and
any row stride; tokens are int32 with -1 (or anything outside of [0, columns)) for "no token".
Work is enqueued on torch's current stream of that GPU, outputs are new tensors of that stream.
There is no fallback: without the library, or off the GPU, every call raises.
"""

import ctypes

import torch

from . import _lib
from ._lib import PGCError, PGC_OK

PGC_F32, PGC_BF16, PGC_F16 = 0, 1, 2

_P, _I32, _I64, _F64, _SIZE = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t


class pgc_dropout_args(ctypes.Structure):
    _fields_ = [("x", _P), ("residual", _P), ("out", _P), ("row_ids", _P), ("rows", _I64), ("cols", _I64),
                ("x_stride", _I64), ("residual_stride", _I64), ("out_stride", _I64), ("first_row", _I64),
                ("seed", ctypes.c_uint64), ("p", _F64), ("dtype", _I32)]


class pgc_logits(ctypes.Structure):
    _fields_ = [("data", _P), ("rows", _I64), ("cols", _I64), ("stride", _I64), ("dtype", _I32)]


class pgc_preference_args(ctypes.Structure):
    _fields_ = [("targets", _P), ("offsets", _P), ("ref_logprobs", _P), ("pair_weights", _P), ("pairs", _I64),
                ("beta", _F64), ("label_smoothing", _F64), ("scale", _F64), ("loss", _P), ("margins", _P),
                ("logprobs", _P), ("dlogits", _P), ("dlogits_stride", _I64)]


class pgc_policy_args(ctypes.Structure):
    _fields_ = [("targets", _P), ("old_logprobs", _P), ("advantages", _P), ("ref_logprobs", _P),
                ("token_weights", _P), ("clip_low", _F64), ("clip_high", _F64), ("kl", _F64), ("scale", _F64),
                ("loss", _P), ("logprobs", _P), ("dlogits", _P), ("dlogits_stride", _I64)]


_SIGNATURES = {
    "pgc_ops_last_error": (ctypes.c_char_p, []),
    "pgc_dropout": (ctypes.c_int, [ctypes.POINTER(pgc_dropout_args), _P]),
    "pgc_dropout_backward": (ctypes.c_int, [ctypes.POINTER(pgc_dropout_args), _P]),
    "pgc_token_logprobs": (ctypes.c_int, [ctypes.POINTER(pgc_logits), _P, _P, _P, _P]),
    "pgc_token_logprobs_backward": (ctypes.c_int, [ctypes.POINTER(pgc_logits), _P, _P, _P, _P, _I64, _P]),
    "pgc_preference_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(pgc_logits), _I64, ctypes.POINTER(_SIZE)]),
    "pgc_preference_loss": (ctypes.c_int, [ctypes.POINTER(pgc_logits), ctypes.POINTER(pgc_preference_args),
                                           _P, _SIZE, _P]),
    "pgc_policy_loss": (ctypes.c_int, [ctypes.POINTER(pgc_logits), ctypes.POINTER(pgc_policy_args), _P]),
}

_DTYPES = {torch.float32: PGC_F32, torch.bfloat16: PGC_BF16, torch.float16: PGC_F16}

_handle = None


def lib():
    """The loaded library with this module's entry points typed."""
    global _handle
    if _handle is None:
        handle = _lib.lib()
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _handle = handle
    return _handle


def exported_symbols():
    return list(_SIGNATURES)


def _check(status):
    if status != PGC_OK:
        raise PGCError(status, lib().pgc_ops_last_error().decode() or lib().pgc_strerror(status).decode())


def _matrix(name, x, like=None):
    """Row stride of a 2-D GPU matrix; of `like`'s shape, type and GPU where given."""
    shape = x.shape
    if like is not None:
        if shape != like.shape or x.dtype != like.dtype or x.device != like.device:
            raise ValueError("%s must have the shape, dtype and device %s, %s, %s"
                             % (name, tuple(like.shape), like.dtype, like.device))
    elif len(shape) != 2 or x.dtype not in _DTYPES or not x.is_cuda:
        raise ValueError("%s must be a 2-D float32, bfloat16 or float16 tensor on the GPU" % name)
    rows, cols = shape
    stride, step = x.stride()
    if step != 1 and cols > 1:
        raise ValueError("the columns of %s must be adjacent" % name)
    if rows <= 1:
        return cols
    if stride < cols:
        raise ValueError("the rows of %s must not overlap" % name)
    return stride


def _array(name, x, like, dtype, shape):
    """Address of a contiguous array on the GPU of `like`; None for none."""
    if x is None:
        return None
    if x.dtype != dtype or x.shape != shape or x.device != like.device or not x.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s"
                         % (name, dtype, tuple(shape), like.device))
    return x.data_ptr()


def _call(like, name, *args):
    """Calls an entry point on torch's current stream of the GPU that `like` is on."""
    fn = getattr(_handle or lib(), name)
    index = like.device.index
    if index == torch.cuda.current_device():
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status != PGC_OK:
        _check(status)


def _raw_stream(index):
    """Handle of torch's current stream of a GPU."""
    return torch.cuda.current_stream(index).cuda_stream


# The same without a Stream object around it, where torch has that (2 us of a call's 12 less).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


def _output(like, out):
    """The tensor that receives a result of `like`'s shape, and its row stride."""
    if out is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format), like.shape[1]
    stride = _matrix("out", out, like)
    if not out.is_inference():
        torch.autograd.graph.increment_version(out)   # autograd notices a saved tensor that this changes
    return out, stride


# ---- dropout ----------------------------------------------------------------------------

def _dropout(name, x, p, seed, residual, row_ids, first_row, out):
    stride = _matrix("x", x)
    rows, cols = x.shape
    out, out_stride = _output(x, out)
    ids = _array("row_ids", row_ids, x, torch.int64, (rows,))
    args = pgc_dropout_args(x.data_ptr(), None if residual is None else residual.data_ptr(), out.data_ptr(), ids,
                            rows, cols, stride, 0 if residual is None else _matrix("residual", residual, x),
                            out_stride, first_row, int(seed) & 0xFFFFFFFFFFFFFFFF, p, _DTYPES[x.dtype])
    _call(x, name, ctypes.byref(args))
    return out


def dropout(x, p, seed, residual=None, row_ids=None, first_row=0, out=None):
    """residual + dropout(x): values of x are kept with probability 1 - p and scaled by its inverse.

    The mask is a function of `seed`, a row's number and the column alone, so that every worker
    that evaluates a sample draws the same one.  A row's number is row_ids[i] (int64) or
    first_row + i.  Use another seed for each step and layer (pgc_splitmix64(seed, t)).
    `out` may be x or residual (not under autograd).
    """
    if torch.is_grad_enabled() and (x.requires_grad or residual is not None and residual.requires_grad):
        if out is not None:
            raise ValueError("out cannot be given where a gradient is asked for")
        return _Dropout.apply(x, residual, p, seed, row_ids, first_row)
    return _dropout("pgc_dropout", x, p, seed, residual, row_ids, first_row, out)


def dropout_backward(dout, p, seed, row_ids=None, first_row=0, out=None):
    """Gradient of dropout's x from the gradient of its output (the residual's is dout itself)."""
    return _dropout("pgc_dropout_backward", dout, p, seed, None, row_ids, first_row, out)


# ---- token log-probabilities --------------------------------------------------------------

def _logits(logits, targets):
    """The logits' description and the targets' address."""
    stride = _matrix("logits", logits)
    rows, cols = logits.shape
    return (pgc_logits(logits.data_ptr(), rows, cols, stride, _DTYPES[logits.dtype]),
            _array("targets", targets, logits, torch.int32, (rows,)))


def token_logprobs(logits, targets):
    """(logprobs [rows], stats [rows, 2]): each row's log-probability of its target, and its maximum
    and the log of its sum of exp(z - maximum), which the backward pass takes."""
    if torch.is_grad_enabled() and logits.requires_grad:
        return _TokenLogprobs.apply(logits, targets)
    return _token_logprobs(logits, targets)


def _token_logprobs(logits, targets):
    z, y = _logits(logits, targets)
    logprobs = logits.new_empty(z.rows, dtype=torch.float32)
    stats = logits.new_empty((z.rows, 2), dtype=torch.float32)
    _call(logits, "pgc_token_logprobs", ctypes.byref(z), y, logprobs.data_ptr(), stats.data_ptr())
    return logprobs, stats


def token_logprobs_backward(logits, targets, stats, grad, out=None):
    """Gradient of the logits from the gradient of the log-probabilities.  `out` may be the logits."""
    z, y = _logits(logits, targets)
    stats = _array("stats", stats, logits, torch.float32, (z.rows, 2))
    grad = _array("grad", grad, logits, torch.float32, (z.rows,))
    out, stride = _output(logits, out)
    _call(logits, "pgc_token_logprobs_backward", ctypes.byref(z), y, stats, grad, out.data_ptr(), stride)
    return out


# ---- losses ---------------------------------------------------------------------------------

def preference_workspace_bytes(logits, pairs):
    """Bytes of the workspace that preference_loss needs for such logits and so many pairs."""
    rows, cols = logits.shape
    return _workspace_bytes(pgc_logits(None, rows, cols, cols, _DTYPES[logits.dtype]), pairs)


def _workspace_bytes(z, pairs):
    out = _SIZE()
    _check(lib().pgc_preference_workspace_bytes(ctypes.byref(z), pairs, ctypes.byref(out)))
    return out.value


def preference_loss(logits, targets, offsets, ref_logprobs=None, beta=0.1, label_smoothing=0.0, scale=1.0,
                    pair_weights=None, gradient=True, out=None, workspace=None):
    """(loss [pairs], margins [pairs], logprobs [rows], dlogits) of the preference loss.

    Sequence q holds the rows [offsets[q], offsets[q + 1]) (int32); pair i prefers sequence 2 i to
    2 i + 1.  dlogits is the gradient of scale * sum(pair_weights * loss), None with gradient=False.
    `out` receives it and may be the logits.  `workspace` (uint8, preference_workspace_bytes(logits,
    pairs)) is allocated where it is not given.
    """
    z, y = _logits(logits, targets)
    pairs = (offsets.numel() - 1) // 2
    offsets = _array("offsets", offsets, logits, torch.int32, (2 * max(pairs, 0) + 1,))
    ref = _array("ref_logprobs", ref_logprobs, logits, torch.float32, (z.rows,))
    weights = _array("pair_weights", pair_weights, logits, torch.float32, (pairs,))
    nbytes = _workspace_bytes(z, pairs) if workspace is None else workspace.numel()
    if workspace is None and nbytes > 0:
        workspace = logits.new_empty(nbytes, dtype=torch.uint8)
    ws = None if workspace is None else _array("workspace", workspace, logits, torch.uint8, workspace.shape)
    loss = logits.new_empty(pairs, dtype=torch.float32)
    margins = logits.new_empty(pairs, dtype=torch.float32)
    logprobs = logits.new_empty(z.rows, dtype=torch.float32)
    stride = 0
    if gradient:
        out, stride = _output(logits, out)
    args = pgc_preference_args(y, offsets, ref, weights, pairs, beta, label_smoothing, scale, loss.data_ptr(),
                               margins.data_ptr(), logprobs.data_ptr(), out.data_ptr() if gradient else None, stride)
    _call(logits, "pgc_preference_loss", ctypes.byref(z), ctypes.byref(args), ws, nbytes)
    return loss, margins, logprobs, out if gradient else None


def policy_loss(logits, targets, old_logprobs, advantages, ref_logprobs=None, clip_low=0.2, clip_high=0.2, kl=0.0,
                scale=1.0, token_weights=None, gradient=True, out=None):
    """(loss [rows], logprobs [rows], dlogits) of the clipped policy loss with a KL term.

    dlogits is the gradient of scale * sum(token_weights * loss), None with gradient=False.  `out`
    receives it and may be the logits.
    """
    z, y = _logits(logits, targets)
    f32, rows = torch.float32, (z.rows,)
    old = _array("old_logprobs", old_logprobs, logits, f32, rows)
    adv = _array("advantages", advantages, logits, f32, rows)
    ref = _array("ref_logprobs", ref_logprobs, logits, f32, rows)
    weights = _array("token_weights", token_weights, logits, f32, rows)
    loss = logits.new_empty(rows, dtype=f32)
    logprobs = logits.new_empty(rows, dtype=f32)
    stride = 0
    if gradient:
        out, stride = _output(logits, out)
    args = pgc_policy_args(y, old, adv, ref, weights, clip_low, clip_high, kl, scale, loss.data_ptr(),
                           logprobs.data_ptr(), out.data_ptr() if gradient else None, stride)
    _call(logits, "pgc_policy_loss", ctypes.byref(z), ctypes.byref(args))
    return loss, logprobs, out if gradient else None


# ---- autograd -------------------------------------------------------------------------------

class _Dropout(torch.autograd.Function):
    """Linear in x and residual, so the gradient is a dropout that has one itself."""

    @staticmethod
    def forward(ctx, x, residual, p, seed, row_ids, first_row):
        ctx.args = p, seed, first_row
        ctx.save_for_backward(row_ids)
        return _dropout("pgc_dropout", x, p, seed, residual, row_ids, first_row, None)

    @staticmethod
    def backward(ctx, dout):
        dx = None
        if ctx.needs_input_grad[0]:
            p, seed, first_row = ctx.args
            dx = dropout(dout.contiguous(), p, seed, row_ids=ctx.saved_tensors[0], first_row=first_row)
        return dx, dout if ctx.needs_input_grad[1] else None, None, None, None, None


class _TokenLogprobs(torch.autograd.Function):
    """The stats carry no gradient."""

    @staticmethod
    def forward(ctx, logits, targets):
        logprobs, stats = _token_logprobs(logits, targets)
        ctx.save_for_backward(logits, targets, stats)
        ctx.mark_non_differentiable(stats)
        return logprobs, stats

    @staticmethod
    def backward(ctx, grad, _):
        logits, targets, stats = ctx.saved_tensors
        return _TokenLogprobsGradient.apply(logits, targets, stats, grad.contiguous()), None


class _TokenLogprobsGradient(torch.autograd.Function):
    """A gradient that has none itself: a graph of it can be made, but not gone back through."""

    @staticmethod
    def forward(ctx, logits, targets, stats, grad):
        return token_logprobs_backward(logits, targets, stats, grad)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("the gradient of token_logprobs is not differentiable")
