"""Operators of neural word models: layer norm, the gated layer, the softmax
cross entropy over a vocabulary, word embedding, the gated recurrence over
documents and distillation from a teacher's top words, each with its backward
pass.

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
MAX_TOP, MAX_LISTED, RECUR_ROWS = 256, 1 << 28, 16

# Every symbol include/lda_ops.h declares.
EXPORTS = ("lda_layer_norm", "lda_layer_norm_backward_workspace", "lda_layer_norm_backward", "lda_gated_workspace",
           "lda_gated", "lda_gated_backward_workspace", "lda_gated_backward", "lda_softmax_xent_workspace",
           "lda_softmax_xent", "lda_softmax_xent_backward_workspace", "lda_softmax_xent_backward", "lda_embedding",
           "lda_embedding_backward_workspace", "lda_embedding_backward", "lda_recurrence_workspace", "lda_recurrence",
           "lda_recurrence_backward_workspace", "lda_recurrence_backward", "lda_recurrence_step",
           "lda_softmax_distill_workspace", "lda_softmax_distill", "lda_softmax_distill_backward_workspace",
           "lda_softmax_distill_backward")


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


class EmbedArgs(ctypes.Structure):
    _fields_ = [("dtype", _I32), ("rows", _I64), ("width", _I32), ("vocab", _I32), ("scale", _F32), ("words", _P),
                ("weight", _P), ("ld_weight", _I64), ("y", _P), ("ldy", _I64), ("dy", _P), ("lddy", _I64),
                ("dweight", _P), ("workspace", _P), ("workspace_bytes", _SIZE), ("stream", _P)]


class RecurArgs(ctypes.Structure):
    _fields_ = [("dtype", _I32), ("rows", _I64), ("cols", _I32), ("docs", _I64), ("offsets", _P), ("x", _P),
                ("ldx", _I64), ("gate", _P), ("ld_gate", _I64), ("state", _P), ("h", _P), ("ldh", _I64), ("last", _P),
                ("kept", _P), ("dh", _P), ("lddh", _I64), ("dlast", _P), ("dx", _P), ("lddx", _I64), ("dgate", _P),
                ("ld_dgate", _I64), ("dstate", _P), ("workspace", _P), ("workspace_bytes", _SIZE), ("stream", _P)]


class DistillArgs(ctypes.Structure):
    _fields_ = [("dtype", _I32), ("rows", _I64), ("width", _I32), ("vocab", _I32), ("top", _I32),
                ("temperature", _F32), ("x", _P), ("ldx", _I64), ("weight", _P), ("ld_weight", _I64), ("bias", _P),
                ("words", _P), ("ld_words", _I64), ("scores", _P), ("ld_scores", _I64), ("loss", _P), ("lse", _P),
                ("logits", _P), ("dloss", _P), ("dx", _P), ("lddx", _I64), ("dweight", _P), ("dbias", _P),
                ("workspace", _P), ("workspace_bytes", _SIZE), ("stream", _P)]


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


def _matrix(name, t, like=None, shape=None, dtype=None):
    """A device matrix with unit column stride, of the type (or ``dtype``) and device of ``like``."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError("%s must be a matrix" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on a HIP device" % name)
    if dtype is not None:
        if t.dtype != dtype or t.get_device() != like.get_device():
            raise ValueError("%s must be %s on the device of x" % (name, dtype))
    elif like is not None:
        if t.dtype != like.dtype or t.get_device() != like.get_device():
            raise ValueError("%s must have the type and device of x" % name)
    elif t.dtype not in _DTYPES:
        raise ValueError("%s must be float32, bfloat16 or float16" % name)
    cols = t.shape[1]
    if shape is not None and t.shape != shape:
        raise ValueError("%s must be %d x %d" % (name, shape[0], shape[1]))
    if cols < 1:
        raise ValueError("%s must have columns" % name)
    if cols > 1 and t.stride(1) != 1:
        raise ValueError("%s must have unit column stride" % name)
    if t.requires_grad:
        _refuse_autograd(name, t)
    return t


def _vector(name, t, like, length, dtype):
    if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.shape[0] != length:
        raise ValueError("%s must be a vector of %d" % (name, length))
    if t.dtype != dtype or t.get_device() != like.get_device():
        raise ValueError("%s must be %s on the device of x" % (name, dtype))
    if length > 1 and t.stride(0) != 1:
        raise ValueError("%s must be contiguous" % name)
    if t.requires_grad:
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


def embedding(words, weight, scale: float = 1.0):
    """``scale * weight[words]`` for int32 ``words``; a row of zeros for a word outside [0, len(weight))."""
    _matrix("weight", weight)
    if not isinstance(words, torch.Tensor) or words.dim() != 1:
        raise ValueError("words must be a vector")
    rows, (vocab, width) = words.shape[0], weight.shape
    _vector("words", words, weight, rows, torch.int32)
    if vocab < 1:
        raise ValueError("weight must have rows")
    y = torch.empty(rows, width, dtype=weight.dtype, device=weight.device)
    a = EmbedArgs(dtype=_DTYPES[weight.dtype], rows=rows, width=width, vocab=vocab, scale=scale,
                  words=words.data_ptr(), weight=weight.data_ptr(), ld_weight=weight.stride(0), y=y.data_ptr(),
                  ldy=width)
    _call("lda_embedding", a, weight.device, workspace=False)
    return y


def embedding_backward(dy, words, vocab: int, scale: float = 1.0):
    """Gradient of :func:`embedding` by the weight, ``vocab`` rows of the type of ``dy``; zero for words without rows."""
    _matrix("dy", dy)
    rows, width = dy.shape
    _vector("words", words, dy, rows, torch.int32)
    if not 1 <= vocab <= MAX_VOCAB:
        raise ValueError("vocab must be 1 to %d" % MAX_VOCAB)
    dweight = torch.empty(vocab, width, dtype=dy.dtype, device=dy.device)
    a = EmbedArgs(dtype=_DTYPES[dy.dtype], rows=rows, width=width, vocab=vocab, scale=scale, words=words.data_ptr(),
                  dy=dy.data_ptr(), lddy=dy.stride(0), dweight=dweight.data_ptr())
    _call("lda_embedding_backward", a, dy.device)
    return dweight


def _state(name, t, like, docs, cols):
    """A state of each document, float32 and contiguous."""
    _matrix(name, t, like, (docs, cols), torch.float32)
    if docs > 1 and t.stride(0) != cols:
        raise ValueError("%s must be contiguous" % name)
    return t


def _recur_args(x, gate, offsets, state):
    _matrix("x", x)
    rows, cols = x.shape
    _matrix("gate", gate, x, x.shape)
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("offsets must be a vector of the documents' number and one more")
    docs = offsets.shape[0] - 1
    _vector("offsets", offsets, x, docs + 1, torch.int64)
    if state is not None:
        _state("state", state, x, docs, cols)
    return RecurArgs(dtype=_DTYPES[x.dtype], rows=rows, cols=cols, docs=docs, offsets=offsets.data_ptr(),
                     x=x.data_ptr(), ldx=x.stride(0), gate=gate.data_ptr(), ld_gate=gate.stride(0),
                     state=None if state is None else state.data_ptr())


def recurrence(x, gate, offsets, state=None):
    """Gated linear recurrence over documents; returns ``(h, last, kept)``.

    Document s has the rows ``offsets[s]`` to ``offsets[s + 1] - 1`` (int64, on
    the device) and begins with ``state[s]`` (float32, or None for 0).  In each
    column ``h_t = f h_{t-1} + (1 - f) x_t`` with ``f = sigmoid(gate_t)``; ``last``
    is the documents' last state in float32, ``kept`` what the backward pass
    takes.  Rows of no document (padding) are 0, whatever they hold.  The offsets
    must not decrease; that is not checked.
    """
    a = _recur_args(x, gate, offsets, state)
    h = torch.empty(a.rows, a.cols, dtype=x.dtype, device=x.device)
    last = torch.empty(a.docs, a.cols, dtype=torch.float32, device=x.device)
    kept = torch.empty(-(-a.rows // RECUR_ROWS), a.cols, dtype=torch.float32, device=x.device)
    a.h, a.ldh, a.last, a.kept = h.data_ptr(), a.cols, last.data_ptr(), kept.data_ptr()
    _call("lda_recurrence", a, x.device)
    return h, last, kept


def recurrence_backward(dh, x, gate, offsets, kept, state=None, dlast=None):
    """Gradients ``(dx, dgate, dstate)`` of :func:`recurrence` for ``dh`` and ``dlast`` (float32, or None for 0).

    ``kept`` is the forward's; ``dstate`` is None where ``state`` is.
    """
    a = _recur_args(x, gate, offsets, state)
    _matrix("dh", dh, x, x.shape)
    _state("kept", kept, x, -(-a.rows // RECUR_ROWS), a.cols)
    if dlast is not None:
        _state("dlast", dlast, x, a.docs, a.cols)
        a.dlast = dlast.data_ptr()
    dx, dgate = (torch.empty(a.rows, a.cols, dtype=x.dtype, device=x.device) for _ in range(2))
    dstate = None if state is None else torch.empty_like(state, memory_format=torch.contiguous_format)
    a.kept, a.dh, a.lddh = kept.data_ptr(), dh.data_ptr(), dh.stride(0)
    a.dx, a.lddx, a.dgate, a.ld_dgate = dx.data_ptr(), a.cols, dgate.data_ptr(), a.cols
    a.dstate = None if dstate is None else dstate.data_ptr()
    _call("lda_recurrence_backward", a, x.device)
    return dx, dgate, dstate


def recurrence_step(x, gate, state, out=None):
    """One row more of each document: ``(h, state)`` from x and gate (a row a document) and the states (float32).

    The new states are written to ``out`` if it is given, which may be ``state`` itself.
    """
    _matrix("x", x)
    rows, cols = x.shape
    _matrix("gate", gate, x, x.shape)
    _state("state", state, x, rows, cols)
    if out is None:
        out = torch.empty(rows, cols, dtype=torch.float32, device=x.device)
    else:
        _state("out", out, x, rows, cols)
        if 0 < abs(out.data_ptr() - state.data_ptr()) < 4 * rows * cols:
            raise ValueError("out must be state or apart from it")
    h = torch.empty(rows, cols, dtype=x.dtype, device=x.device)
    a = RecurArgs(dtype=_DTYPES[x.dtype], rows=rows, cols=cols, docs=rows, x=x.data_ptr(), ldx=x.stride(0),
                  gate=gate.data_ptr(), ld_gate=gate.stride(0), state=state.data_ptr(), h=h.data_ptr(), ldh=cols,
                  last=out.data_ptr())
    _call("lda_recurrence_step", a, x.device, workspace=False)
    return h, out


def _distill_args(x, weight, words, scores, bias, temperature):
    _matrix("x", x)
    _matrix("weight", weight, x)
    rows, width = x.shape
    vocab = weight.shape[0]
    if vocab < 1 or weight.shape[1] != width:
        raise ValueError("weight must have rows of %d columns" % width)
    if not isinstance(words, torch.Tensor) or words.dim() != 2 or not 1 <= words.shape[1] <= MAX_TOP:
        raise ValueError("words must be a matrix of 1 to %d columns" % MAX_TOP)
    top = words.shape[1]
    _matrix("words", words, x, (rows, top), torch.int32)
    _matrix("scores", scores, x, (rows, top), torch.float32)
    if bias is not None:
        _vector("bias", bias, x, vocab, torch.float32)
    return DistillArgs(dtype=_DTYPES[x.dtype], rows=rows, width=width, vocab=vocab, top=top, temperature=temperature,
                       x=x.data_ptr(), ldx=x.stride(0), weight=weight.data_ptr(), ld_weight=weight.stride(0),
                       bias=None if bias is None else bias.data_ptr(), words=words.data_ptr(),
                       ld_words=words.stride(0), scores=scores.data_ptr(), ld_scores=scores.stride(0))


def softmax_distill(x, weight, words, scores, bias=None, temperature: float = 1.0):
    """How far the softmax over ``(x @ weight.T + bias) / temperature`` is from a teacher's, per row.

    The teacher lists ``words`` (int32 ids, [rows, top]; outside [0, vocab) an
    empty place) and their ``scores`` (float32 logits, or logarithms of
    probabilities); its softmax over ``scores / temperature`` is taken over the
    listed words of a row.  Returns ``(loss, lse, logits)`` in float32: the
    Kullback-Leibler divergence from the teacher, the log-sum-exp, and the logits
    of the listed words (0 at empty places).  A row without words, or whose
    scores are all -inf, has loss 0.  A bias of -inf masks a word.  The other
    logits are not kept.
    """
    a = _distill_args(x, weight, words, scores, bias, temperature)
    loss, lse = torch.empty(2, a.rows, dtype=torch.float32, device=x.device).unbind(0)
    logits = torch.empty(a.rows, a.top, dtype=torch.float32, device=x.device)
    a.loss, a.lse, a.logits = loss.data_ptr(), lse.data_ptr(), logits.data_ptr()
    _call("lda_softmax_distill", a, x.device)
    return loss, lse, logits


def softmax_distill_backward(dloss, lse, logits, x, weight, words, scores, bias=None, temperature: float = 1.0):
    """Gradients ``(dx, dweight, dbias)`` of :func:`softmax_distill` for ``dloss`` (float32, one per row).

    ``lse`` and ``logits`` are the forward's; ``dbias`` is None where ``bias`` is.
    The teacher gets no gradient.
    """
    a = _distill_args(x, weight, words, scores, bias, temperature)
    _vector("lse", lse, x, a.rows, torch.float32)
    _vector("dloss", dloss, x, a.rows, torch.float32)
    _state("logits", logits, x, a.rows, a.top)
    dx = torch.empty(a.rows, a.width, dtype=x.dtype, device=x.device)
    dweight = torch.empty(a.vocab, a.width, dtype=x.dtype, device=x.device)
    dbias = None if bias is None else torch.empty_like(bias)
    a.lse, a.logits, a.dloss = lse.data_ptr(), logits.data_ptr(), dloss.data_ptr()
    a.dx, a.lddx, a.dweight = dx.data_ptr(), a.width, dweight.data_ptr()
    a.dbias = None if dbias is None else dbias.data_ptr()
    _call("lda_softmax_distill_backward", a, x.device)
    return dx, dweight, dbias
