"""Operators on the way from a worker's samples to its local gradient (binding of the calls in ``include/laq.h``).

The library's own models end at 16 classes and one hidden layer; a larger model's gradients come from outside
(``MODEL_EXTERNAL``, ``Laq.set_gradients``).  These are the pieces such a model needs beside the quantizer:

``linear`` / ``linear_backward``                     a layer's product with bias, activation and residual; its gradient
``token_logprobs`` / ``token_logprobs_backward``     log probabilities of given tokens, entropy, top alternatives; gradient
``distill`` / ``distill_backward``                   divergence from a teacher's top logits; gradient, alone or with the loss
``gated`` / ``gated_backward``                       a gated feed-forward block's two projections and their product; its gradient
``pack8`` / ``unpack8``                              a matrix in 8 bits with a scale for each block of 128 (``Packed8``), and back:
                                                     activations that the gradients above read in that form
``linear8``                                          a layer's product on two such matrices

Tensors are CUDA tensors with unit stride within a row and any row stride; outputs are allocated here unless ``out`` is
given, which is refused if it shares memory with another tensor of the call other than where a call says so.  Gradients
are calls of their own: none of this takes part in torch's autograd.  Calls run on ``stream`` (default: the current stream
of the tensors' device) and do not synchronise: their inputs must be ready in that stream's order, and may be let go of as
soon as the call has returned.  They launch kernels only: there is no CPU fallback.  ``check_status`` reports a bounded wait
of the product kernels that ran out.
"""
import collections
import ctypes as C
import threading

import torch

from . import laq
from .laq import LAQ_OK, LAQ_ETIMEOUT, LAQ_EWORKSPACE, LaqError

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
LINEAR_STARVE = 1

_status = {}        # per device: the word in which the product kernels record a bounded wait that ran out
_failures = {}      # per device: how often the word was found set, and cleared
_status_lock = threading.Lock()


def _refuse(message):
    raise ValueError(message)


# These checks run on every call, whose kernel may take a few microseconds: they use the cheapest forms of the questions.
_current_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream
_local = threading.local()          # the calling thread's buffer for error texts, and the failures that it has been told of


def _check(t, name, index=None, dtype=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse("%s must be a CUDA tensor" % name)
    if index is not None and t.get_device() != index:
        _refuse("%s is on %s, the other tensors on cuda:%d" % (name, t.device, index))
    if dtype is not None and t.dtype is not dtype:
        _refuse("%s must be %s, not %s" % (name, dtype, t.dtype))


def _rows(t, name, index=None, dtype=None, shape=None):
    """A matrix with unit stride within its rows: (pointer, row stride, rows, columns)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or (index is not None and t.get_device() != index) or (dtype is not None and t.dtype is not dtype):
        _check(t, name, index, dtype)
    size = t.shape
    if len(size) != 2:
        _refuse("%s must have two dimensions" % name)
    rows, cols = size
    if shape is not None and (rows, cols) != shape:
        _refuse("%s must have shape %s, not %s" % (name, shape, (rows, cols)))
    stride, within = t.stride()
    if within != 1 and cols > 1:
        _refuse("%s must have unit stride within a row" % name)
    if rows <= 1:
        stride = cols
    elif stride < cols:
        _refuse("the rows of %s overlap" % name)
    return t.data_ptr(), stride, rows, cols


def _table(rows, cols, dtype, device):
    return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)


def _vector(t, name, index, dtype, n):
    """A contiguous vector of n elements, or None: its pointer."""
    if t is None:
        return None
    _check(t, name, index, dtype)
    if t.dim() != 1 or t.shape[0] != n:
        _refuse("%s must have shape (%d,), not %s" % (name, n, tuple(t.shape)))
    if n > 1 and t.stride(0) != 1:
        _refuse("%s must be contiguous" % name)
    return t.data_ptr()


def _on(index, stream, body, *tensors):
    """body(raw stream) with the tensors' device current; outputs that it allocates belong to that stream.  `tensors` are those
    that the caller has given: their memory is not handed out again before a stream of the call's own has done with it."""
    if stream is None:
        if _current_device() == index:
            return body(_raw_stream(index))
        with torch.cuda.device(index):
            return body(_raw_stream(index))
    if stream.device.index != index:
        _refuse("the stream belongs to %s, the tensors to cuda:%d" % (stream.device, index))
    with torch.cuda.stream(stream):
        result = body(stream.cuda_stream)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return result


def _errors():
    err = getattr(_local, "err", None)
    if err is None:
        err = _local.err = C.create_string_buffer(256)
    return err


def _call(function, *args):
    err = _errors()
    rc = function(*args, err, 256)
    if rc != LAQ_OK:
        raise LaqError(rc, err.value.decode())


def _logits(logits):
    ptr, stride, T, V = _rows(logits, "logits")
    dtype = DTYPES.get(logits.dtype)
    if dtype is None:
        _refuse("logits must be float32, bfloat16 or float16")
    if V < 1:
        _refuse("logits have no columns")
    return (ptr, dtype, T, V, stride), T, logits.get_device()


def token_logprobs(logits, tokens=None, top_k=0, temperature=1.0, stream=None):
    """Log probabilities of ``tokens`` [rows] int32 under softmax(logits / temperature), with the rows' entropies, their
    lse and, for top_k > 0, the top_k most likely tokens (ties: lowest index).

    Returns a dict: logprob, entropy, lse [rows] float32, and top_tokens [rows, top_k] int32 with top_logprobs float32.
    Without ``tokens`` there is no logprob.  A negative token leaves its row out: zeros and no alternatives.
    """
    head, T, index = _logits(logits)
    tok = _vector(tokens, "tokens", index, torch.int32, T)
    if not 0 <= top_k <= 32:
        _refuse("top_k must be 0..32")

    def body(raw):
        dev = logits.device
        stats = _table(3, T, torch.float32, dev)
        p = stats.data_ptr()
        logprob, entropy, lse = stats.unbind(0)
        out = dict(entropy=entropy, lse=lse) if tok is None else dict(logprob=logprob, entropy=entropy, lse=lse)
        tp = vp = None
        if top_k:
            out["top_tokens"] = a = _table(T, top_k, torch.int32, dev)
            out["top_logprobs"] = b = _table(T, top_k, torch.float32, dev)
            tp, vp = a.data_ptr(), b.data_ptr()
        _call(laq.load_library().laq_token_logprobs, *head, temperature, tok, top_k, None if tok is None else p, p + 4 * T,
              p + 8 * T, tp, vp, raw)
        return out

    return _on(index, stream, body, logits, tokens)


def _gradient_out(logits, out):
    if out is None:
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    ptr, stride, _, _ = _rows(out, "out", logits.get_device(), logits.dtype, tuple(logits.shape))
    return out, ptr, stride


def token_logprobs_backward(logits, tokens, lse, entropy=None, d_logprob=None, d_entropy=None, temperature=1.0, out=None,
                            stream=None):
    """Gradient with respect to the logits of sum(d_logprob * logprob + d_entropy * entropy), given lse and entropy as
    ``token_logprobs`` returned them.  ``out`` may be ``logits`` itself."""
    head, T, index = _logits(logits)
    if tokens is None or lse is None:
        _refuse("tokens and lse are needed")
    if d_entropy is not None and entropy is None:
        _refuse("the gradient of the entropy needs the entropy")
    f32 = torch.float32
    ptrs = (_vector(tokens, "tokens", index, torch.int32, T), _vector(lse, "lse", index, f32, T),
            _vector(entropy, "entropy", index, f32, T), _vector(d_logprob, "d_logprob", index, f32, T),
            _vector(d_entropy, "d_entropy", index, f32, T))

    def body(raw):
        dx, dptr, dstride = _gradient_out(logits, out)
        _call(laq.load_library().laq_token_logprobs_backward, *head, temperature, *ptrs, dptr, dstride, raw)
        return dx

    return _on(index, stream, body, logits, tokens, lse, entropy, d_logprob, d_entropy, out)


def _teacher(tokens, values, index, T):
    tp, ts, rows, k = _rows(tokens, "teacher_tokens", index, torch.int32)
    if rows != T:
        _refuse("teacher_tokens must have a row for every row of the logits")
    vp, vs, _, _ = _rows(values, "teacher_logits", index, torch.float32, (rows, k))
    if ts != vs:
        _refuse("teacher_tokens and teacher_logits must have the same row stride")
    if not 1 <= k <= 128:
        _refuse("the teacher must have 1..128 entries per row")
    return tp, vp, k, ts


def distill(logits, teacher_tokens, teacher_logits, temperature=1.0, d_loss=None, out=None, stream=None):
    """Divergence of the student's softmax(logits / temperature) from a teacher known by its top logits: teacher_tokens
    [rows, k] int32 (negative: no entry) and teacher_logits [rows, k] float32, k <= 128.

    Returns a dict: loss and lse [rows] float32.  With ``d_loss`` [rows] float32, the gradient of whatever the losses are
    summed into, the same call also returns dlogits (in ``out`` if given, which may be ``logits`` itself).
    """
    head, T, index = _logits(logits)
    teacher = _teacher(teacher_tokens, teacher_logits, index, T)
    dl = _vector(d_loss, "d_loss", index, torch.float32, T)
    if d_loss is None and out is not None:
        _refuse("out without d_loss")

    def body(raw):
        stats = _table(2, T, torch.float32, logits.device)
        p = stats.data_ptr()
        loss, lse = stats.unbind(0)
        res = dict(loss=loss, lse=lse)
        dptr, dstride = None, 0
        if d_loss is not None:
            res["dlogits"], dptr, dstride = _gradient_out(logits, out)
        _call(laq.load_library().laq_distill, *head, temperature, *teacher, p, p + 4 * T, dl, dptr, dstride, raw)
        return res

    return _on(index, stream, body, logits, teacher_tokens, teacher_logits, d_loss, out)


def distill_backward(logits, teacher_tokens, teacher_logits, lse, d_loss, temperature=1.0, out=None, stream=None):
    """The gradient of ``distill`` for a d_loss that is only known after the loss; lse as ``distill`` returned it."""
    head, T, index = _logits(logits)
    teacher = _teacher(teacher_tokens, teacher_logits, index, T)
    if lse is None or d_loss is None:
        _refuse("lse and d_loss are needed")
    ptrs = (_vector(lse, "lse", index, torch.float32, T), _vector(d_loss, "d_loss", index, torch.float32, T))

    def body(raw):
        dx, dptr, dstride = _gradient_out(logits, out)
        _call(laq.load_library().laq_distill_backward, *head, temperature, *teacher, *ptrs, dptr, dstride, raw)
        return dx

    return _on(index, stream, body, logits, teacher_tokens, teacher_logits, lse, d_loss, out)


# --- the layer -------------------------------------------------------------------------------------------------------

def _status_word(index):
    word = _status.get(index)
    if word is None:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("call ops.init(device) before the first capture of a linear call on a device")
        word = torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", index))
        torch.cuda.synchronize(index)        # other streams may use it from now on
        word = _status.setdefault(index, word)
    seen = _seen()
    if index not in seen:                    # this thread answers for what happens from now on
        with _status_lock:
            seen[index] = _failures.get(index, 0)
    return word


def _seen():
    seen = getattr(_local, "seen", None)
    if seen is None:
        seen = _local.seen = {}
    return seen


def _device_index(device):
    """The GPU that a device argument names: None and "cuda" are the current one."""
    if device is None:
        return torch.cuda.current_device()
    device = torch.device(device)
    if device.type != "cuda":
        _refuse("%s is not a CUDA device" % device)
    return torch.cuda.current_device() if device.index is None else device.index


def init(device=None):
    """Set up the device's status word (done by the first linear call otherwise, which must then not be captured)."""
    index = _device_index(device)
    with torch.cuda.device(index):
        _status_word(index)


def check_status(device=None):
    """Synchronises the device and raises LAQ_ETIMEOUT if a bounded wait of a linear call on it, of any thread, ran out since
    this thread's last check (its first call on the device, if it has not checked before).  A wait that ran out is told to
    every thread that checks, whichever finds it first: all of them share the device's status word."""
    index = _device_index(device)
    word = _status.get(index)
    if word is None:
        return
    seen = _seen()
    with _status_lock:
        torch.cuda.synchronize(index)
        bits = int(word.item())
        if bits:
            _failures[index] = _failures.get(index, 0) + 1       # before it is cleared: what comes between belongs to it
            word.zero_()
            torch.cuda.synchronize(index)
        told, seen[index] = seen.get(index, 0), _failures.get(index, 0)
    if told != seen[index]:
        raise LaqError(LAQ_ETIMEOUT, "a bounded wait inside a product kernel ran out%s: outputs since the last check are not "
                                     "complete" % (" (bits %d)" % bits if bits else ""))


def _activation(name):
    act = ACTIVATIONS.get(name)
    if act is None:
        _refuse("activation must be one of %s" % ", ".join(sorted(ACTIVATIONS)))
    return act


def _layer_call(x, weight, activation, flags, index):
    c = laq.laq_linear_call()
    c.x, c.ld_x, c.M, c.K = _rows(x, "x")
    c.w, c.ld_w, c.N, inputs = _rows(weight, "weight", index, x.dtype)
    if x.dtype is not torch.bfloat16 and x.dtype is not torch.float16:
        _refuse("x must be bfloat16 or float16")
    if inputs != c.K:
        _refuse("weight must be [outputs, %d]" % c.K)
    act = _activation(activation)
    if c.K < 1 or c.N < 1:
        _refuse("a layer needs inputs and outputs")
    c.dtype, c.activation, c.flags = DTYPES[x.dtype], act, flags
    return c


def _result(out, rows, cols, dtype, index, device):
    """`out` or a new matrix: (matrix, pointer, row stride)."""
    if out is None:
        out = _table(rows, cols, dtype, device)
        return out, out.data_ptr(), cols
    ptr, stride, _, _ = _rows(out, "out", index, dtype, (rows, cols))
    return out, ptr, stride


def _forward(function, need, call, more, odd, workspace, index, raw):
    """A call that needs no workspace unless its operands lie at odd addresses: one is made if the call asks for it, which it does
    before it launches anything, or at once where they do."""
    if workspace is None and not odd:
        err = _errors()
        rc = function(call, *more, None, 0, raw, err, 256)
        if rc == LAQ_OK:
            return
        if rc != LAQ_EWORKSPACE:
            raise LaqError(rc, err.value.decode())
    ws, wp, wn = _workspace(need(call, *more, 0), index, workspace)
    _call(function, call, *more, wp, wn, raw)


def _workspace(need, index, given):
    if need == 0:
        return None, None, 0
    if given is None:
        given = torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", index))
    else:
        _check(given, "workspace", index, torch.uint8)
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
    _check(x, "x")
    index, dt = x.get_device(), x.dtype
    c = _layer_call(x, weight, activation, flags, index)
    shape = (c.M, c.N)
    c.bias = _vector(bias, "bias", index, dt, c.N)
    if residual is not None:
        c.residual, c.ld_residual, _, _ = _rows(residual, "residual", index, dt, shape)

    def body(raw):
        c.status = _status_word(index).data_ptr()
        y = _table(*shape, dt, x.device) if out is None else out
        c.y, c.ld_y, _, _ = _rows(y, "out", index, dt, shape)
        z = None
        if preact:
            z = _table(*shape, dt, x.device)
            c.z, c.ld_z = z.data_ptr(), c.N
        ws, wp, wn = _workspace(L.laq_linear_workspace_bytes(C.byref(c), 0), index, workspace)
        _call(L.laq_linear_forward, C.byref(c), wp, wn, raw)
        return (y, z) if preact else y

    return _on(index, stream, body, x, weight, bias, residual, out, workspace)


def linear_backward(dy, x, weight, z=None, activation="none", dx=True, dw=True, db=True, dw_dtype=None, workspace=None,
                    stream=None, flags=0):
    """Gradient of ``linear`` for dy [rows, outputs]; z as linear(preact=True) returned it (not needed for activation none).  Any of
    x, weight and z may be a ``Packed8``: the gradient is then that of the layer on the values it stands for.  Those of x and weight are
    taken in dy's type, as ``unpack8`` gives them: exact in bfloat16; in float16 those beyond 65504 are 65504, and below 2^-21 they
    are rounded to multiples of 2^-24.  z is read as it is.

    Returns a dict with those of dx [rows, inputs], dw [outputs, inputs] and db [outputs] float32 that are asked for.
    dw_dtype is the layer's type (default) or float32, the latter for activations none and relu.  The residual's gradient
    is dy.
    """
    L = laq.load_library()
    packed = isinstance(x, Packed8) or isinstance(weight, Packed8) or isinstance(z, Packed8)
    typed = dy if packed else x
    _check(typed, "dy" if packed else "x")
    index, dt = typed.get_device(), typed.dtype
    dw_dtype = dt if dw_dtype is None else dw_dtype
    if dw and dw_dtype is not dt and dw_dtype is not torch.float32:
        _refuse("dw_dtype must be %s or float32" % dt)
    xq = wq = zq = None
    if packed:
        c = laq.laq_linear_call()
        c.dtype, c.activation, c.flags = _layer_type(dt, "dy"), _activation(activation), flags
        c.x, c.ld_x, c.M, c.K, xq = _rows_or_codes(x, "x", index, dt)
        c.w, c.ld_w, c.N, inputs, wq = _rows_or_codes(weight, "weight", index, dt)
        if inputs != c.K:
            _refuse("weight must be [outputs, %d]" % c.K)
        if c.K < 1 or c.N < 1:
            _refuse("a layer needs inputs and outputs")
    else:
        c = _layer_call(x, weight, activation, flags, index)
    c.dy, c.ld_dy, _, _ = _rows(dy, "dy", index, dt, (c.M, c.N))
    if activation != "none":
        if z is None:
            _refuse("the gradient of an activation needs z")
        c.z, c.ld_z, _, _, zq = _rows_or_codes(z, "z", index, dt, (c.M, c.N))

    def body(raw):
        c.status = _status_word(index).data_ptr()
        dev, res = dy.device, {}
        if dx:
            res["dx"] = t = _table(c.M, c.K, dt, dev)
            c.dx, c.ld_dx = t.data_ptr(), c.K
        if dw:
            res["dw"] = t = _table(c.N, c.K, dw_dtype, dev)
            c.dw, c.ld_dw, c.dw_dtype = t.data_ptr(), c.K, DTYPES[dw_dtype]
        if db:
            res["db"] = t = torch.empty(c.N, dtype=torch.float32, device=dev)
            c.db = t.data_ptr()
        if packed:
            ws, wp, wn = _workspace(L.laq_linear_blocks_workspace_bytes(C.byref(c), xq, wq, 1), index, workspace)
            _call(L.laq_linear_blocks_backward, C.byref(c), xq, wq, zq, wp, wn, raw)
        else:
            ws, wp, wn = _workspace(L.laq_linear_workspace_bytes(C.byref(c), 1), index, workspace)
            _call(L.laq_linear_backward, C.byref(c), wp, wn, raw)
        return res

    return _on(index, stream, body, dy, *_tensors(x), *_tensors(weight), *_tensors(z), workspace)


# --- 8 bits ----------------------------------------------------------------------------------------------------------

class Packed8(collections.namedtuple("Packed8", ("codes", "scales"))):
    """A matrix in 8 bits: codes [rows, cols] float8_e4m3fn (unit stride within a row) and scales float32, either
    [rows, ceil(cols / 128)], a scale for each 128 columns of a row, or [ceil(rows / 128), ceil(cols / 128)], a scale for each
    tile of 128 rows and 128 columns.  It stands for codes * scales."""
    __slots__ = ()

    @property
    def shape(self):
        return self.codes.shape


BLOCK = 128


def _layer_type(dtype, name):
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        _refuse("%s must be bfloat16 or float16" % name)
    return DTYPES[dtype]


def _packed(p, name, index=None, shape=None):
    """A Packed8: (laq_blocks, rows, columns)."""
    if not isinstance(p, Packed8):
        _refuse("%s must be a Packed8" % name)
    codes, scales = p
    pc, ld_codes, rows, cols = _rows(codes, name + ".codes", index, torch.float8_e4m3fn, shape)
    ps, ld_scales, down, across = _rows(scales, name + ".scales", codes.get_device(), torch.float32)
    if across != -(-cols // BLOCK) or (down != rows and down != -(-rows // BLOCK)):
        _refuse("%s.scales must have shape %s or %s, not %s" % (name, (rows, -(-cols // BLOCK)), (-(-rows // BLOCK), -(-cols // BLOCK)),
                                                               (down, across)))
    return laq.laq_blocks(pc, ld_codes, ps, ld_scales, 1 if down == rows else BLOCK), rows, cols


def _rows_or_codes(t, name, index, dtype, shape=None):
    """A matrix of the layer's type or a Packed8: (pointer, row stride, rows, columns, laq_blocks or None)."""
    if isinstance(t, Packed8):
        q, rows, cols = _packed(t, name, index, shape)
        return None, cols, rows, cols, q
    return *_rows(t, name, index, dtype, shape), None


def _tensors(t):
    return tuple(t) if isinstance(t, Packed8) else (t,)


def _new_packed(rows, cols, tiles, device):
    """An uninitialised Packed8 and its laq_blocks; rows of codes begin 16 bytes apart or multiples of that, as the product reads
    them best."""
    pitch, across = -(-cols // 16) * 16, -(-cols // BLOCK)
    codes = torch.empty_strided((rows, cols), (pitch, 1), dtype=torch.float8_e4m3fn, device=device)
    scales = _table(-(-rows // BLOCK) if tiles else rows, across, torch.float32, device)
    return Packed8(codes, scales), laq.laq_blocks(codes.data_ptr(), pitch, scales.data_ptr(), across, BLOCK if tiles else 1)


def pack8(x, tiles=False, out=None, stream=None):
    """x [rows, cols] (float32, bfloat16 or float16) in 8 bits: a ``Packed8`` with a scale for each 128 columns of a row or, with
    tiles=True (weights), for each tile of 128 x 128.

    A scale is the least power of two that brings its block's largest finite value within 448, so that a value is off by half a
    step of its code alone: 2^-4 of it, or 2^-10 of the scale below 2^-6 of that.  NaN and infinities become NaN.  ``out`` is a
    Packed8 to write to.
    """
    ptr, stride, rows, cols = _rows(x, "x")
    index, dtype = x.get_device(), DTYPES.get(x.dtype)
    if dtype is None:
        _refuse("x must be float32, bfloat16 or float16")
    if cols < 1:
        _refuse("x has no columns")

    def body(raw):
        if out is None:
            p, q = _new_packed(rows, cols, tiles, x.device)
        else:
            p, (q, _, _) = out, _packed(out, "out", index, (rows, cols))
            if rows > 1 and (q.block_rows != 1) != bool(tiles):
                _refuse("out.scales are not those of tiles=%s" % bool(tiles))
        _call(laq.load_library().laq_pack_blocks, ptr, dtype, rows, cols, stride, C.byref(q), raw)
        return p

    return _on(index, stream, body, x, *_tensors(out))


def unpack8(packed, dtype=torch.bfloat16, out=None, stream=None):
    """The values of a ``Packed8`` in dtype (float32, bfloat16 or float16), rounded to the nearest; finite values beyond its
    largest are that.  Values that ``pack8`` wrote are exact in float32 and bfloat16."""
    q, rows, cols = _packed(packed, "packed")
    index = packed.codes.get_device()
    if out is not None:
        _check(out, "out", index)
        dtype = out.dtype
    code = DTYPES.get(dtype)
    if code is None:
        _refuse("dtype must be float32, bfloat16 or float16")
    if cols < 1:
        _refuse("packed has no columns")

    def body(raw):
        if out is None:
            t = _table(rows, cols, dtype, packed.codes.device)
            ptr, stride = t.data_ptr(), cols
        else:
            t, (ptr, stride, _, _) = out, _rows(out, "out", index, dtype, (rows, cols))
        _call(laq.load_library().laq_unpack_blocks, C.byref(q), rows, cols, ptr, code, stride, raw)
        return t

    return _on(index, stream, body, *packed, out)


def linear8(x, weight, bias=None, activation="none", residual=None, preact=False, dtype=torch.bfloat16, out=None, workspace=None,
            stream=None, flags=0):
    """``linear`` on operands in 8 bits: x [rows, inputs] a ``Packed8`` with a scale for each 128 columns of a row, weight
    [outputs, inputs] one with a scale for each tile (``pack8(w, tiles=True)``); bias, residual and results in dtype, bfloat16 or
    float16.  Its gradient is ``linear_backward`` with the same x and weight.  This call reads any code times any scale; that one takes x
    and weight in dtype, so that in float16, where values lie beyond its range, it is not the gradient of what was computed here."""
    L = laq.load_library()
    xq, M, K = _packed(x, "x")
    index = x.codes.get_device()
    wq, N, inputs = _packed(weight, "weight", index)
    c = laq.laq_linear_call()
    c.dtype, c.activation, c.flags = _layer_type(dtype, "dtype"), _activation(activation), flags
    if inputs != K:
        _refuse("weight must be [outputs, %d]" % K)
    if K < 1 or N < 1:
        _refuse("a layer needs inputs and outputs")
    if M > 1 and xq.block_rows != 1:
        _refuse("x must have a scale for each row")
    if N > 1 and wq.block_rows != BLOCK:
        _refuse("weight must have a scale for each tile of 128 rows")
    c.M, c.N, c.K = M, N, K
    c.bias = _vector(bias, "bias", index, dtype, N)
    if residual is not None:
        c.residual, c.ld_residual, _, _ = _rows(residual, "residual", index, dtype, (M, N))

    def body(raw):
        c.status = _status_word(index).data_ptr()
        y, c.y, c.ld_y = _result(out, M, N, dtype, index, x.codes.device)
        z = None
        if preact:
            z = _table(M, N, dtype, x.codes.device)
            c.z, c.ld_z = z.data_ptr(), N
        _forward(L.laq_linear_blocks_forward, L.laq_linear_blocks_workspace_bytes, C.byref(c), (C.byref(xq), C.byref(wq)),
                 ((xq.codes or 0) | (xq.ld_codes if M > 1 else 0) | wq.codes | (wq.ld_codes if N > 1 else 0)) & 15, workspace, index, raw)
        return (y, z) if preact else y

    return _on(index, stream, body, *x, *weight, bias, residual, out, workspace)


# --- the gated block -------------------------------------------------------------------------------------------------

def _gated_call(weight, M, K, activation, flags, index, dtype):
    c = laq.laq_gated_call()
    c.dtype, c.activation, c.flags = _layer_type(dtype, "x"), _activation(activation), flags
    c.w, c.ld_w, rows, inputs = _rows(weight, "weight", index, dtype)
    if inputs != K or rows % 2:
        _refuse("weight must be [2 gates, %d]" % K)
    if K < 1 or rows < 2:
        _refuse("a block needs inputs and gates")
    c.M, c.F, c.K = M, rows // 2, K
    return c


def gated(x, weight, bias=None, activation="silu", preact=False, out=None, workspace=None, stream=None, flags=0):
    """act(g) * u for the two halves g and u [rows, gates] of z = x weight^T + bias: x [rows, inputs], weight [2 gates, inputs] (the
    gates' rows first), bias [2 gates], all bfloat16 or all float16; at most 65536 inputs.

    Returns h [rows, gates], or (h, z) for preact=True, z [rows, 2 gates], and for preact="packed", z in 8 bits, which is
    ``pack8`` of the former.  ``gated_backward`` takes either.
    """
    L = laq.load_library()
    ptr, ld, M, K = _rows(x, "x")
    index, dt = x.get_device(), x.dtype
    c = _gated_call(weight, M, K, activation, flags, index, dt)
    c.x, c.ld_x = ptr, ld
    N = 2 * c.F
    c.bias = _vector(bias, "bias", index, dt, N)
    if preact not in (False, True, "packed"):
        _refuse("preact must be False, True or \"packed\"")

    def body(raw):
        c.status = _status_word(index).data_ptr()
        h, c.h, c.ld_h = _result(out, M, N // 2, dt, index, x.device)
        z = None
        if preact == "packed":
            z, q = _new_packed(M, N, False, x.device)
            c.z_blocks = C.pointer(q)
        elif preact:
            z = _table(M, N, dt, x.device)
            c.z, c.ld_z = z.data_ptr(), N
        _forward(L.laq_gated_forward, L.laq_gated_workspace_bytes, C.byref(c), (), ((c.x or 0) | c.ld_x * 2 | c.w | c.ld_w * 2) & 15, workspace, index, raw)
        return (h, z) if preact else h

    return _on(index, stream, body, x, weight, bias, out, workspace)


def gated_backward(dh, x, weight, z, activation="silu", dx=True, dw=True, db=True, workspace=None, stream=None, flags=0):
    """Gradient of ``gated`` for dh [rows, gates]; z as gated(preact=True) or gated(preact="packed") returned it, x as it was or
    packed (``pack8``; taken in dh's type as by ``linear_backward``).  The gradient of z is rounded to dh's type before the two products:
    in float16 a product of dh and a gate or an up beyond 65504 is infinite there, and dx and dw with it (db is not).

    Returns a dict with those of dx [rows, inputs], dw [2 gates, inputs] and db [2 gates] float32 that are asked for.
    """
    L = laq.load_library()
    _check(dh, "dh")
    index, dt = dh.get_device(), dh.dtype
    ptr, ld, M, K, xq = _rows_or_codes(x, "x", index, dt)
    c = _gated_call(weight, M, K, activation, flags, index, dt)
    c.x, c.ld_x = ptr, ld
    N = 2 * c.F
    c.dh, c.ld_dh, _, _ = _rows(dh, "dh", index, dt, (M, c.F))
    c.z, c.ld_z, _, _, zq = _rows_or_codes(z, "z", index, dt, (M, N))
    if xq is not None:
        c.x_blocks = C.pointer(xq)
    if zq is not None:
        c.z_blocks = C.pointer(zq)

    def body(raw):
        c.status = _status_word(index).data_ptr()
        dev, res = dh.device, {}
        if dx:
            res["dx"] = t = _table(M, K, dt, dev)
            c.dx, c.ld_dx = t.data_ptr(), K
        if dw:
            res["dw"] = t = _table(N, K, dt, dev)
            c.dw, c.ld_dw = t.data_ptr(), K
        if db:
            res["db"] = t = torch.empty(N, dtype=torch.float32, device=dev)
            c.db = t.data_ptr()
        ws, wp, wn = _workspace(L.laq_gated_workspace_bytes(C.byref(c), 1), index, workspace)
        _call(L.laq_gated_backward, C.byref(c), wp, wn, raw)
        return res

    return _on(index, stream, body, dh, *_tensors(x), weight, *_tensors(z), workspace)
