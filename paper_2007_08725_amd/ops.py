"""Operators of neural word models: layer norm, the gated layer and the softmax
cross entropy over a vocabulary, each with its backward pass.

Thin ctypes binding over the operators of ``liblda.so`` (``include/lda_ops.h``):
it checks and marshals torch tensors, allocates outputs and workspaces with
torch's caching allocator and enqueues on torch's current stream.  Every
operator runs in the library's HIP kernels; there is no CPU fallback.

Matrices are float32, bfloat16 or float16, one type per call, with unit column
stride; rows may be strided.  Results are the same bits on every run.

The operators are no part of torch's autograd graph: gradients come from the
``_backward`` calls.  Tensors that require a gradient are refused while autograd
records (``ValueError``); call under ``torch.no_grad()`` or on detached tensors.
"""
from __future__ import annotations

import ctypes

import torch

from . import LDA_OK, LDAError, load_library

_P, _I32, _I64, _F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
_SIZE = ctypes.c_size_t
_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"silu": 0, "gelu": 1, "sigmoid": 2}
MAX_ROWS, MAX_COLS, MAX_VOCAB, MAX_TILES = 1 << 24, 1 << 20, 1 << 24, 1 << 23

# Every symbol include/lda_ops.h declares.
EXPORTS = ("lda_layer_norm", "lda_layer_norm_backward_workspace", "lda_layer_norm_backward", "lda_gated_workspace",
           "lda_gated", "lda_gated_backward_workspace", "lda_gated_backward", "lda_softmax_xent_workspace",
           "lda_softmax_xent", "lda_softmax_xent_backward_workspace", "lda_softmax_xent_backward")


class NormArgs(ctypes.Structure):
    _fields_ = [("dtype", _I32), ("rows", _I64), ("cols", _I32), ("eps", _F32), ("x", _P), ("ldx", _I64),
                ("weight", _P), ("bias", _P), ("y", _P), ("ldy", _I64), ("mean", _P), ("rstd", _P), ("dy", _P),
                ("lddy", _I64), ("dx", _P), ("lddx", _I64), ("dweight", _P), ("dbias", _P), ("workspace", _P),
                ("workspace_bytes", _SIZE), ("stream", _P)]


class GatedArgs(ctypes.Structure):
    _fields_ = [("dtype", _I32), ("act", _I32), ("rows", _I64), ("width", _I32), ("hidden", _I32), ("x", _P),
                ("ldx", _I64), ("w_gate", _P), ("ld_gate", _I64), ("w_value", _P), ("ld_value", _I64), ("h", _P),
                ("ldh", _I64), ("dh", _P), ("lddh", _I64), ("dx", _P), ("lddx", _I64), ("dw_gate", _P),
                ("dw_value", _P), ("workspace", _P), ("workspace_bytes", _SIZE), ("stream", _P)]


class XentArgs(ctypes.Structure):
    _fields_ = [("dtype", _I32), ("rows", _I64), ("width", _I32), ("vocab", _I32), ("x", _P), ("ldx", _I64),
                ("weight", _P), ("ld_weight", _I64), ("bias", _P), ("labels", _P), ("loss", _P), ("lse", _P),
                ("dloss", _P), ("dx", _P), ("lddx", _I64), ("dweight", _P), ("dbias", _P), ("workspace", _P),
                ("workspace_bytes", _SIZE), ("stream", _P)]


_functions = {}


def _function(name):
    fn = _functions.get(name)
    if fn is None:
        fn = getattr(load_library(), name)
        fn.restype = ctypes.c_int
        fn.argtypes = [_P, _P] if name.endswith("_workspace") else [_P]
        _functions[name] = fn
    return fn


def _call(name, args, device, workspace=True):
    """Size the workspace, allocate it and call the operator on the current stream of ``device``."""
    if torch.cuda.current_device() != device.index:
        with torch.cuda.device(device):
            return _call(name, args, device, workspace)
    args.stream = torch._C._cuda_getCurrentRawStream(device.index)
    scratch = None
    if workspace:
        size = _SIZE()
        _check(_function(name + "_workspace")(ctypes.byref(args), ctypes.byref(size)))
        if size.value:
            # freed to torch's allocator on return: it hands the memory out again on this stream only
            scratch = torch.empty(size.value, dtype=torch.uint8, device=device)
            args.workspace = scratch.data_ptr()
            args.workspace_bytes = size.value
    _check(_function(name)(ctypes.byref(args)))


def _check(status):
    if status != LDA_OK:
        raise LDAError(status, load_library().lda_last_error(None).decode())


def _refuse_autograd(name, t):
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, which torch would not get: call the operator under torch.no_grad() "
                         "and its _backward" % name)


def _matrix(name, t, like=None, shape=None):
    """A device matrix with unit column stride, of the type and device of ``like``."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a matrix" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on a HIP device" % name)
    if t.dtype not in _DTYPES:
        raise ValueError("%s must be float32, bfloat16 or float16" % name)
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError("%s must have the type and device of x" % name)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %d x %d" % (name, shape[0], shape[1]))
    if t.shape[1] < 1:
        raise ValueError("%s must have columns" % name)
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("%s must have unit column stride" % name)
    _refuse_autograd(name, t)
    return t


def _vector(name, t, like, length, dtype):
    if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.shape[0] != length:
        raise ValueError("%s must be a vector of %d" % (name, length))
    if t.dtype != dtype or t.device != like.device:
        raise ValueError("%s must be %s on the device of x" % (name, dtype))
    if length > 1 and t.stride(0) != 1:
        raise ValueError("%s must be contiguous" % name)
    _refuse_autograd(name, t)
    return t


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    """Layer norm of each row of ``x``; returns ``(y, mean, rstd)``, the statistics in float32 for the backward pass.

    ``weight`` and ``bias`` are given together or not at all.
    """
    _matrix("x", x)
    rows, cols = x.shape
    if (weight is None) != (bias is None):
        raise ValueError("weight and bias must be given together")
    if weight is not None:
        _vector("weight", weight, x, cols, x.dtype)
        _vector("bias", bias, x, cols, x.dtype)
    y = torch.empty(rows, cols, dtype=x.dtype, device=x.device)
    mean, rstd = torch.empty(2, rows, dtype=torch.float32, device=x.device).unbind(0)
    a = NormArgs(dtype=_DTYPES[x.dtype], rows=rows, cols=cols, eps=eps, x=x.data_ptr(), ldx=x.stride(0),
                 weight=None if weight is None else weight.data_ptr(), bias=None if bias is None else bias.data_ptr(),
                 y=y.data_ptr(), ldy=cols, mean=mean.data_ptr(), rstd=rstd.data_ptr())
    _call("lda_layer_norm", a, x.device, workspace=False)
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd):
    """Gradients ``(dx, dweight, dbias)`` of :func:`layer_norm`; the last two are None where ``weight`` is."""
    _matrix("x", x)
    rows, cols = x.shape
    _matrix("dy", dy, x, x.shape)
    _vector("mean", mean, x, rows, torch.float32)
    _vector("rstd", rstd, x, rows, torch.float32)
    a = NormArgs(dtype=_DTYPES[x.dtype], rows=rows, cols=cols, x=x.data_ptr(), ldx=x.stride(0), mean=mean.data_ptr(),
                 rstd=rstd.data_ptr(), dy=dy.data_ptr(), lddy=dy.stride(0))
    dx = torch.empty(rows, cols, dtype=x.dtype, device=x.device)
    a.dx, a.lddx = dx.data_ptr(), cols
    dweight = dbias = None
    if weight is not None:
        _vector("weight", weight, x, cols, x.dtype)
        dweight, dbias = torch.empty_like(weight), torch.empty_like(weight)
        a.weight, a.dweight, a.dbias = weight.data_ptr(), dweight.data_ptr(), dbias.data_ptr()
    _call("lda_layer_norm_backward", a, x.device)
    return dx, dweight, dbias


def _gated_args(x, w_gate, w_value, act):
    _matrix("x", x)
    if act not in ACTIVATIONS:
        raise ValueError("act must be one of %s" % ", ".join(ACTIVATIONS))
    _matrix("w_gate", w_gate, x)
    hidden = w_gate.shape[0]
    if hidden < 1 or w_gate.shape[1] != x.shape[1]:
        raise ValueError("w_gate must have rows of %d columns" % x.shape[1])
    _matrix("w_value", w_value, x, w_gate.shape)
    return GatedArgs(dtype=_DTYPES[x.dtype], act=ACTIVATIONS[act], rows=x.shape[0], width=x.shape[1], hidden=hidden,
                     x=x.data_ptr(), ldx=x.stride(0), w_gate=w_gate.data_ptr(), ld_gate=w_gate.stride(0),
                     w_value=w_value.data_ptr(), ld_value=w_value.stride(0))


def gated(x, w_gate, w_value, act: str = "silu"):
    """``act(x @ w_gate.T) * (x @ w_value.T)``; ``act`` is "silu", "gelu" (with the error function) or "sigmoid"."""
    a = _gated_args(x, w_gate, w_value, act)
    h = torch.empty(a.rows, a.hidden, dtype=x.dtype, device=x.device)
    a.h, a.ldh = h.data_ptr(), a.hidden
    _call("lda_gated", a, x.device)
    return h


def gated_backward(dh, x, w_gate, w_value, act: str = "silu"):
    """Gradients ``(dx, dw_gate, dw_value)`` of :func:`gated`, which are recomputed from ``x`` (nothing is kept)."""
    a = _gated_args(x, w_gate, w_value, act)
    _matrix("dh", dh, x, (a.rows, a.hidden))
    dx = torch.empty(a.rows, a.width, dtype=x.dtype, device=x.device)
    dw_gate = torch.empty(a.hidden, a.width, dtype=x.dtype, device=x.device)
    dw_value = torch.empty_like(dw_gate)
    a.dh, a.lddh = dh.data_ptr(), dh.stride(0)
    a.dx, a.lddx = dx.data_ptr(), a.width
    a.dw_gate, a.dw_value = dw_gate.data_ptr(), dw_value.data_ptr()
    _call("lda_gated_backward", a, x.device)
    return dx, dw_gate, dw_value


def _xent_args(x, weight, labels, bias):
    _matrix("x", x)
    _matrix("weight", weight, x)
    rows, width = x.shape
    vocab = weight.shape[0]
    if vocab < 1 or weight.shape[1] != width:
        raise ValueError("weight must have rows of %d columns" % width)
    _vector("labels", labels, x, rows, torch.int32)
    if bias is not None:
        _vector("bias", bias, x, vocab, torch.float32)
    return XentArgs(dtype=_DTYPES[x.dtype], rows=rows, width=width, vocab=vocab, x=x.data_ptr(), ldx=x.stride(0),
                    weight=weight.data_ptr(), ld_weight=weight.stride(0),
                    bias=None if bias is None else bias.data_ptr(), labels=labels.data_ptr())


def softmax_xent(x, weight, labels, bias=None):
    """Loss per row of the softmax over ``x @ weight.T + bias`` and its log-sum-exp, ``(loss, lse)`` in float32.

    ``labels`` are int32 word ids; a label outside [0, vocab) leaves its row out
    (loss 0).  ``bias`` is float32 or None; -inf masks a word.  The logits are
    not kept.
    """
    a = _xent_args(x, weight, labels, bias)
    loss, lse = torch.empty(2, a.rows, dtype=torch.float32, device=x.device).unbind(0)
    a.loss, a.lse = loss.data_ptr(), lse.data_ptr()
    _call("lda_softmax_xent", a, x.device)
    return loss, lse


def softmax_xent_backward(dloss, lse, x, weight, labels, bias=None):
    """Gradients ``(dx, dweight, dbias)`` of :func:`softmax_xent` for ``dloss`` (float32, one per row).

    ``lse`` is the forward's; ``dbias`` is None where ``bias`` is.
    """
    a = _xent_args(x, weight, labels, bias)
    _vector("lse", lse, x, a.rows, torch.float32)
    _vector("dloss", dloss, x, a.rows, torch.float32)
    dx = torch.empty(a.rows, a.width, dtype=x.dtype, device=x.device)
    dweight = torch.empty(a.vocab, a.width, dtype=x.dtype, device=x.device)
    dbias = None if bias is None else torch.empty_like(bias)
    a.lse, a.dloss = lse.data_ptr(), dloss.data_ptr()
    a.dx, a.lddx, a.dweight = dx.data_ptr(), a.width, dweight.data_ptr()
    a.dbias = None if dbias is None else dbias.data_ptr()
    _call("lda_softmax_xent_backward", a, x.device)
    return dx, dweight, dbias
