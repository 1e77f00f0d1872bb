"""Operators that turn a language model's outputs into a partition's loss and gradient.

Binding of include/pgc_ops.h (through binding/pgc_ops_torch.cpp), which states what each operator computes: dropout with a mask
that is a function of seed, row number and column; log-probabilities of given tokens; the
preference loss of pairs of sequences; the clipped policy loss with a KL term.  The losses take
logits and return the loss and the logits' gradient; `logits.backward(dlogits)` carries it on
through a model, and a backward pass through the loss itself raises.  dropout and token_logprobs take part in autograd where an input asks for it (backward;
forward-mode derivatives are refused, and so are traces by torch.jit.trace and make_fx).

`out` must not ask for a gradient itself, unless it is the logits and a model's output.

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


# The C entry points' structures and signatures, for calls by address; calls on tensors go through the compiled module.

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


class _Native:
    """Functions of the compiled module that calls the entry points on torch's tensors; loaded at the
    first call, so that the package can be imported before it is built."""

    def __getattr__(self, name):
        try:
            from . import _ops_torch
        except ImportError as e:
            raise RuntimeError("the compiled binding of the operators is not built (%s); run "
                               "`python -m paper_2607_20739_amd.build`" % e) from e
        for f in ("dropout", "dropout_backward", "token_logprobs", "token_logprobs_backward", "preference_loss",
                  "policy_loss"):
            setattr(self, f, getattr(_ops_torch, f))
        return self.__dict__[name]


_native = _Native()


# ---- dropout ----------------------------------------------------------------------------

def dropout(x, p, seed, residual=None, row_ids=None, first_row=0, out=None):
    """residual + dropout(x): values of x are kept with probability 1 - p and scaled by its inverse.

    The mask is a function of `seed`, a row's number and the column alone, so that every worker
    that evaluates a sample draws the same one.  A row's number is row_ids[i] (int64) or
    first_row + i.  Use another seed for each step and layer (pgc_splitmix64(seed, t)).
    `out` may be x or residual (not under autograd).
    """
    # What is no tensor is left to the binding, which refuses it.
    if torch.is_grad_enabled() and (getattr(x, "requires_grad", False) or
                                    residual is not None and getattr(residual, "requires_grad", False)):
        if out is not None:
            raise ValueError("out cannot be given where a gradient is asked for")
        return _Dropout.apply(x, residual, p, seed, row_ids, first_row)
    return _native.dropout(x, p, int(seed), residual, row_ids, first_row, out)


def dropout_backward(dout, p, seed, row_ids=None, first_row=0, out=None):
    """Gradient of dropout's x from the gradient of its output (the residual's is dout itself)."""
    return _native.dropout_backward(dout, p, int(seed), None, row_ids, first_row, out)


# ---- token log-probabilities --------------------------------------------------------------

def token_logprobs(logits, targets):
    """(logprobs [rows], stats [rows, 2]): each row's log-probability of its target, and its maximum
    and the log of its sum of exp(z - maximum), which the backward pass takes."""
    if torch.is_grad_enabled() and getattr(logits, "requires_grad", False):
        return _TokenLogprobs.apply(logits, targets)
    return _native.token_logprobs(logits, targets)


def token_logprobs_backward(logits, targets, stats, grad, out=None):
    """Gradient of the logits from the gradient of the log-probabilities.  `out` may be the logits."""
    return _native.token_logprobs_backward(logits, targets, stats, grad, out)


# ---- losses ---------------------------------------------------------------------------------

def preference_workspace_bytes(logits, pairs):
    """Bytes of the workspace that preference_loss needs for such logits and so many pairs."""
    if not (torch.is_tensor(logits) and logits.dim() == 2 and logits.dtype in _DTYPES):
        raise ValueError("logits must be a 2-D float32, bfloat16 or float16 tensor")
    rows, cols = logits.shape
    z, out = pgc_logits(None, rows, cols, cols, _DTYPES[logits.dtype]), _SIZE()
    status = lib().pgc_preference_workspace_bytes(ctypes.byref(z), pairs, ctypes.byref(out))
    if status != PGC_OK:
        raise PGCError(status, lib().pgc_ops_last_error().decode())
    return out.value


def preference_loss(logits, targets, offsets, ref_logprobs=None, beta=0.1, label_smoothing=0.0, scale=1.0,
                    pair_weights=None, gradient=True, out=None, workspace=None):
    """(loss [pairs], margins [pairs], logprobs [rows], dlogits) of the preference loss.

    Sequence q holds the rows [offsets[q], offsets[q + 1]) (int32); pair i prefers sequence 2 i to
    2 i + 1.  dlogits is the gradient of scale * sum(pair_weights * loss), None with gradient=False.
    `out` receives it and may be the logits.  `workspace` (uint8, preference_workspace_bytes(logits,
    pairs)) is allocated where it is not given.
    """
    results = _native.preference_loss(logits, targets, offsets, ref_logprobs, beta, label_smoothing, scale, pair_weights,
                                      gradient, out, workspace)
    return _marked(logits, results) if logits.requires_grad else results


def policy_loss(logits, targets, old_logprobs, advantages, ref_logprobs=None, clip_low=0.2, clip_high=0.2, kl=0.0,
                scale=1.0, token_weights=None, gradient=True, out=None):
    """(loss [rows], logprobs [rows], dlogits) of the clipped policy loss with a KL term.

    dlogits is the gradient of scale * sum(token_weights * loss), None with gradient=False.  `out`
    receives it and may be the logits.
    """
    results = _native.policy_loss(logits, targets, old_logprobs, advantages, ref_logprobs, clip_low, clip_high, kl, scale,
                                  token_weights, gradient, out)
    return _marked(logits, results) if logits.requires_grad else results


def _marked(logits, results):
    """Results (dlogits last) for logits that ask for a gradient: in a sum that is differentiated, they raise instead of
    missing in it."""
    if torch.is_grad_enabled():
        return (*_LossWithoutGraph.apply(logits, results[:-1]), results[-1])
    return results


# ---- autograd -------------------------------------------------------------------------------

class _Dropout(torch.autograd.Function):
    """Linear in x and residual, so the gradient is a dropout that has one itself."""

    @staticmethod
    def forward(ctx, x, residual, p, seed, row_ids, first_row):
        ctx.args = p, seed, first_row
        ctx.save_for_backward(row_ids)
        return _native.dropout(x, p, int(seed), residual, row_ids, first_row, None)

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
        logprobs, stats = _native.token_logprobs(logits, targets)
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


class _LossWithoutGraph(torch.autograd.Function):
    """Values whose gradient has been computed already."""

    @staticmethod
    def forward(ctx, logits, values):
        return values

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the losses' gradient is their result dlogits: call logits.backward(dlogits)")
