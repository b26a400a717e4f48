"""Operators on the way from a worker's samples to its local gradient (binding of the calls in ``include/laq.h``).

The library's own models end at 16 classes and one hidden layer; a larger model's gradients come from outside
(``MODEL_EXTERNAL``, ``Laq.set_gradients``).  These are the pieces such a model needs beside the quantizer:

``linear`` / ``linear_backward``                     a layer's product with bias, activation and residual; its gradient
``token_logprobs`` / ``token_logprobs_backward``     log probabilities of given tokens, entropy, top alternatives; gradient
``distill`` / ``distill_backward``                   divergence from a teacher's top logits; gradient, alone or with the loss

Tensors are CUDA tensors with unit stride within a row and any row stride; outputs are allocated here unless ``out`` is
given.  Calls run on ``stream`` (default: the current stream of the tensors' device) and do not synchronise.  They launch
kernels only: there is no CPU fallback.  ``check_status`` reports a bounded wait of the product kernels that ran out.
"""
import ctypes as C

import torch

from . import laq
from .laq import LAQ_OK, LAQ_ETIMEOUT, LaqError

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
LINEAR_STARVE = 1

_status = {}        # per device: the word in which the product kernels record a bounded wait that ran out


def _refuse(message):
    raise ValueError(message)


def _check(t, name, device, dtype=None, shape=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse("%s must be a CUDA tensor" % name)
    if device is not None and t.device != device:
        _refuse("%s is on %s, the other tensors on %s" % (name, t.device, device))
    if dtype is not None and t.dtype != dtype:
        _refuse("%s must be %s, not %s" % (name, dtype, t.dtype))
    if shape is not None and tuple(t.shape) != shape:
        _refuse("%s must have shape %s, not %s" % (name, shape, tuple(t.shape)))
    return t


def _rows(t, name, device=None, dtype=None, shape=None):
    """A matrix with unit stride within its rows: (pointer, row stride)."""
    _check(t, name, device, dtype, shape)
    if t.dim() != 2:
        _refuse("%s must have two dimensions" % name)
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        _refuse("%s must have unit stride within a row" % name)
    stride = t.stride(0) if rows > 1 else cols
    if stride < cols:
        _refuse("the rows of %s overlap" % name)
    return t.data_ptr(), stride


def _vector(t, name, device, dtype, n):
    """A contiguous vector of n elements, or None: its pointer."""
    if t is None:
        return None
    _check(t, name, device, dtype, (n,))
    if n > 1 and t.stride(0) != 1:
        _refuse("%s must be contiguous" % name)
    return t.data_ptr()


class _On:
    """The device of a call made current, and its stream: an output allocated inside belongs to that stream."""

    def __init__(self, device, stream):
        self.device, self.stream, self.guard = device, stream, None

    def __enter__(self):
        if self.stream is not None:
            self.guard = torch.cuda.stream(self.stream)
        elif torch.cuda.current_device() != self.device.index:
            self.guard = torch.cuda.device(self.device)
        if self.guard is not None:
            self.guard.__enter__()
        return self.stream.cuda_stream if self.stream is not None else torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _call(function, *args):
    err = C.create_string_buffer(256)
    rc = function(*args, err, 256)
    if rc != LAQ_OK:
        raise LaqError(rc, err.value.decode())


def _logits(logits):
    ptr, stride = _rows(logits, "logits")
    if logits.dtype not in DTYPES:
        _refuse("logits must be float32, bfloat16 or float16")
    if logits.shape[1] < 1:
        _refuse("logits have no columns")
    return ptr, DTYPES[logits.dtype], logits.shape[0], logits.shape[1], stride


def token_logprobs(logits, tokens=None, top_k=0, temperature=1.0, stream=None):
    """Log probabilities of ``tokens`` [rows] int32 under softmax(logits / temperature), with the rows' entropies, their
    lse and, for top_k > 0, the top_k most likely tokens (ties: lowest index).

    Returns a dict: logprob, entropy, lse [rows] float32, and top_tokens [rows, top_k] int32 with top_logprobs float32.
    Without ``tokens`` there is no logprob.  A negative token leaves its row out: zeros and no alternatives.
    """
    L = laq.load_library()
    head = _logits(logits)
    dev, T = logits.device, logits.shape[0]
    tok = _vector(tokens, "tokens", dev, torch.int32, T)
    if not 0 <= top_k <= 32:
        _refuse("top_k must be 0..32")
    with _On(dev, stream) as st:
        stats = torch.empty((3, T), dtype=torch.float32, device=dev)
        out = dict(logprob=stats[0], entropy=stats[1], lse=stats[2])
        if tokens is None:
            del out["logprob"]
        p = stats.data_ptr()
        if top_k:
            out["top_tokens"] = torch.empty((T, top_k), dtype=torch.int32, device=dev)
            out["top_logprobs"] = torch.empty((T, top_k), dtype=torch.float32, device=dev)
        _call(L.laq_token_logprobs, *head, temperature, tok, top_k, p if tokens is not None else None, p + 4 * T, p + 8 * T,
              out["top_tokens"].data_ptr() if top_k else None, out["top_logprobs"].data_ptr() if top_k else None, st)
    return out


def _gradient_out(logits, out):
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    ptr, stride = _rows(out, "out", logits.device, logits.dtype, tuple(logits.shape))
    return out, ptr, stride


def token_logprobs_backward(logits, tokens, lse, entropy=None, d_logprob=None, d_entropy=None, temperature=1.0, out=None,
                            stream=None):
    """Gradient with respect to the logits of sum(d_logprob * logprob + d_entropy * entropy), given lse and entropy as
    ``token_logprobs`` returned them.  ``out`` may be ``logits`` itself."""
    L = laq.load_library()
    head = _logits(logits)
    dev, T = logits.device, logits.shape[0]
    if tokens is None or lse is None:
        _refuse("tokens and lse are needed")
    ptrs = [_vector(tokens, "tokens", dev, torch.int32, T)]
    ptrs += [_vector(t, name, dev, torch.float32, T) for t, name in
             ((lse, "lse"), (entropy, "entropy"), (d_logprob, "d_logprob"), (d_entropy, "d_entropy"))]
    with _On(dev, stream) as st:
        out, dptr, dstride = _gradient_out(logits, out)
        _call(L.laq_token_logprobs_backward, *head, temperature, *ptrs, dptr, dstride, st)
    return out


def _teacher(tokens, values, device, rows):
    tp, ts = _rows(tokens, "teacher_tokens", device, torch.int32)
    vp, vs = _rows(values, "teacher_logits", device, torch.float32, tuple(tokens.shape))
    if tokens.shape[0] != rows:
        _refuse("teacher_tokens must have a row for every row of the logits")
    if ts != vs:
        _refuse("teacher_tokens and teacher_logits must have the same row stride")
    return tp, vp, tokens.shape[1], ts


def distill(logits, teacher_tokens, teacher_logits, temperature=1.0, d_loss=None, out=None, stream=None):
    """Divergence of the student's softmax(logits / temperature) from a teacher known by its top logits: teacher_tokens
    [rows, k] int32 (negative: no entry) and teacher_logits [rows, k] float32, k <= 128.

    Returns a dict: loss and lse [rows] float32.  With ``d_loss`` [rows] float32, the gradient of whatever the losses are
    summed into, the same call also returns dlogits (in ``out`` if given, which may be ``logits`` itself).
    """
    L = laq.load_library()
    head = _logits(logits)
    dev, T = logits.device, logits.shape[0]
    teacher = _teacher(teacher_tokens, teacher_logits, dev, T)
    dl = _vector(d_loss, "d_loss", dev, torch.float32, T)
    if d_loss is None and out is not None:
        _refuse("out without d_loss")
    with _On(dev, stream) as st:
        stats = torch.empty((2, T), dtype=torch.float32, device=dev)
        res = dict(loss=stats[0], lse=stats[1])
        dptr, dstride = None, 0
        if d_loss is not None:
            res["dlogits"], dptr, dstride = _gradient_out(logits, out)
        p = stats.data_ptr()
        _call(L.laq_distill, *head, temperature, *teacher, p, p + 4 * T, dl, dptr, dstride, st)
    return res


def distill_backward(logits, teacher_tokens, teacher_logits, lse, d_loss, temperature=1.0, out=None, stream=None):
    """The gradient of ``distill`` for a d_loss that is only known after the loss; lse as ``distill`` returned it."""
    L = laq.load_library()
    head = _logits(logits)
    dev, T = logits.device, logits.shape[0]
    teacher = _teacher(teacher_tokens, teacher_logits, dev, T)
    if lse is None or d_loss is None:
        _refuse("lse and d_loss are needed")
    ptrs = [_vector(lse, "lse", dev, torch.float32, T), _vector(d_loss, "d_loss", dev, torch.float32, T)]
    with _On(dev, stream) as st:
        out, dptr, dstride = _gradient_out(logits, out)
        _call(L.laq_distill_backward, *head, temperature, *teacher, *ptrs, dptr, dstride, st)
    return out


# --- the layer -------------------------------------------------------------------------------------------------------

def _status_word(device):
    word = _status.get(device.index)
    if word is None:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("call ops.init(device) before the first capture of a linear call on a device")
        word = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.synchronize(device)       # other streams may use it from now on
        _status[device.index] = word
    return word


def init(device=None):
    """Set up the device's status word (done by the first linear call otherwise, which must then not be captured)."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(device):
        _status_word(torch.device("cuda", torch.cuda.current_device()))


def check_status(device=None):
    """Synchronises the device and raises LAQ_ETIMEOUT if a bounded wait of a linear call ran out since the last check."""
    index = torch.cuda.current_device() if device is None else torch.device(device).index
    word = _status.get(index)
    if word is None:
        return
    torch.cuda.synchronize(index)
    bits = int(word.item())
    if bits:
        word.zero_()
        torch.cuda.synchronize(index)
        raise LaqError(LAQ_ETIMEOUT, "a bounded wait inside a product kernel ran out (bits %d): outputs since the last check "
                                     "are not complete" % bits)


def _layer_call(x, weight, activation, flags):
    c = laq.laq_linear_call()
    c.x, c.ld_x = _rows(x, "x")
    if x.dtype not in (torch.bfloat16, torch.float16):
        _refuse("x must be bfloat16 or float16")
    if weight.dim() != 2 or weight.shape[1] != x.shape[1]:
        _refuse("weight must be [outputs, %d]" % x.shape[1])
    c.w, c.ld_w = _rows(weight, "weight", x.device, x.dtype)
    if activation not in ACTIVATIONS:
        _refuse("activation must be one of %s" % ", ".join(sorted(ACTIVATIONS)))
    if x.shape[1] < 1 or weight.shape[0] < 1:
        _refuse("a layer needs inputs and outputs")
    c.dtype, c.activation = DTYPES[x.dtype], ACTIVATIONS[activation]
    c.M, c.N, c.K, c.flags = x.shape[0], weight.shape[0], x.shape[1], flags
    c.status = _status_word(x.device).data_ptr()
    return c


def _workspace(L, c, backward, device, given):
    need = L.laq_linear_workspace_bytes(C.byref(c), backward)
    if need == 0:
        return None, None, 0
    if given is None:
        given = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        _check(given, "workspace", device, torch.uint8)
        if given.dim() != 1 or not given.is_contiguous():
            _refuse("workspace must be a contiguous vector of bytes")
    return given, given.data_ptr(), given.numel()


def linear(x, weight, bias=None, activation="none", residual=None, preact=False, out=None, workspace=None, stream=None, flags=0):
    """act(x weight^T + bias) + residual for x [rows, inputs], weight [outputs, inputs], bias [outputs], residual
    [rows, outputs], all bfloat16 or all float16; activation none, relu, gelu (tanh form) or silu.

    Returns y, or (y, z) with preact=True, z = x weight^T + bias, which ``linear_backward`` needs where there is an
    activation.  ``out`` may be ``residual`` itself.  ``workspace`` (uint8) replaces the one allocated here, see
    laq_linear_workspace_bytes; calls that may overlap need workspaces of their own.
    """
    L = laq.load_library()
    _rows(x, "x")
    dev, dt = x.device, x.dtype
    with _On(dev, stream) as st:
        c = _layer_call(x, weight, activation, flags)
        shape = (c.M, c.N)
        c.bias = _vector(bias, "bias", dev, dt, c.N)
        if residual is not None:
            c.residual, c.ld_residual = _rows(residual, "residual", dev, dt, shape)
        y = torch.empty(shape, dtype=dt, device=dev) if out is None else out
        c.y, c.ld_y = _rows(y, "out", dev, dt, shape)
        z = None
        if preact:
            z = torch.empty(shape, dtype=dt, device=dev)
            c.z, c.ld_z = z.data_ptr(), c.N
        ws, wp, wn = _workspace(L, c, 0, dev, workspace)
        _call(L.laq_linear_forward, C.byref(c), wp, wn, st)
    return (y, z) if preact else y


def linear_backward(dy, x, weight, z=None, activation="none", dx=True, dw=True, db=True, dw_dtype=None, workspace=None,
                    stream=None, flags=0):
    """Gradient of ``linear`` for dy [rows, outputs]; z as linear(preact=True) returned it (not needed for activation none).

    Returns a dict with those of dx [rows, inputs], dw [outputs, inputs] and db [outputs] float32 that are asked for.
    dw_dtype is the layer's type (default) or float32, the latter for activations none and relu.  The residual's gradient
    is dy.
    """
    L = laq.load_library()
    _rows(x, "x")
    dev, dt = x.device, x.dtype
    dw_dtype = dt if dw_dtype is None else dw_dtype
    if dw and dw_dtype not in (dt, torch.float32):
        _refuse("dw_dtype must be %s or float32" % dt)
    with _On(dev, stream) as st:
        c = _layer_call(x, weight, activation, flags)
        c.dy, c.ld_dy = _rows(dy, "dy", dev, dt, (c.M, c.N))
        if activation != "none":
            if z is None:
                _refuse("the gradient of an activation needs z")
            c.z, c.ld_z = _rows(z, "z", dev, dt, (c.M, c.N))
        out = {}
        if dx:
            out["dx"] = torch.empty((c.M, c.K), dtype=dt, device=dev)
            c.dx, c.ld_dx = out["dx"].data_ptr(), c.K
        if dw:
            out["dw"] = torch.empty((c.N, c.K), dtype=dw_dtype, device=dev)
            c.dw, c.ld_dw, c.dw_dtype = out["dw"].data_ptr(), c.K, DTYPES[dw_dtype]
        if db:
            out["db"] = torch.empty(c.N, dtype=torch.float32, device=dev)
            c.db = out["db"].data_ptr()
        ws, wp, wn = _workspace(L, c, 1, dev, workspace)
        _call(L.laq_linear_backward, C.byref(c), wp, wn, st)
    return out
