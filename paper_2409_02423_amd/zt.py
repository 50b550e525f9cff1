"""Python binding of the training-step operators of libzc (include/zt.h): argument marshalling only.

Every function has the name and meaning of the C entry point it calls.  Tensors are torch CUDA tensors of the
current device, used as device memory; the kernels are enqueued on torch's current stream unless a stream is given, and what a
call allocates (outputs that are not passed, workspaces) belongs to the stream it runs on.  There is no fallback: if the HIP
library cannot be loaded, every call raises.
"""
import ctypes
from array import array

import torch

from . import zc
from .zc import ZC_ERR_CAPACITY, ZC_OK, ZcError  # noqa: F401

ZC_ERR_ARG = -10
ZT_RMS, ZT_LAYER = 0, 1
ZT_GATE_NONE, ZT_GATE_CHANNEL, ZT_GATE_FULL = 0, 1, 2
ZT_MAX_COLS, ZT_MAX_ROWS = 32768, 1 << 30
ZT_SLOTS = 512

EXPORTS = ("zt_residual_norm", "zt_residual_work_bytes", "zt_residual_norm_backward", "zt_sum_squares", "zt_norm", "zt_clip", "zt_adamw")

_DTYPES = {torch.float32: zc.ZC_F32, torch.bfloat16: zc.ZC_BF16, torch.float16: zc.ZC_F16}


class Residual(ctypes.Structure):
    """struct zt_residual"""
    _fields_ = [("rows", ctypes.c_size_t), ("cols", ctypes.c_size_t), ("dtype", ctypes.c_int), ("kind", ctypes.c_int), ("post", ctypes.c_int),
                ("gate", ctypes.c_int), ("residual_scale", ctypes.c_float), ("eps", ctypes.c_float)] + [
                    ("stride_" + name, ctypes.c_size_t) for name in ("x", "b", "gate", "y", "h", "dy", "dh", "dx", "db", "dgate")]


class AdamwForm(ctypes.Structure):
    """struct zt_adamw_form"""
    _fields_ = [("n", ctypes.c_size_t), ("grad_dtype", ctypes.c_int), ("half_dtype", ctypes.c_int), ("step", ctypes.c_longlong),
                ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("scale", ctypes.c_float), ("max_norm", ctypes.c_float), ("d_state", ctypes.c_void_p)]


_lib = None


def lib():
    """The loaded C library (zc.lib()) with these operators' signatures."""
    global _lib
    L = zc.lib()
    if _lib is not L:
        p, size, form = ctypes.c_void_p, ctypes.c_size_t, ctypes.POINTER(Residual)
        L.zt_residual_norm.argtypes = [form] + [p] * 11
        L.zt_residual_work_bytes.restype = size
        L.zt_residual_work_bytes.argtypes = [form]
        L.zt_residual_norm_backward.argtypes = [form] + [p] * 17 + [size, p]
        L.zt_sum_squares.argtypes = [p, p, p, ctypes.c_int, ctypes.c_int, p, p]
        L.zt_norm.argtypes = [p, ctypes.c_float, p, p]
        L.zt_clip.argtypes = [p, p, p, p, p, ctypes.c_int, p, ctypes.c_float, ctypes.c_float, p, p]
        L.zt_adamw.argtypes = [ctypes.POINTER(AdamwForm), p, p, p, p, p, p, p, p]
        _lib = L
    return _lib


def _check(rc, what):
    if rc != ZC_OK:
        raise ZcError(rc, what)


def _empty(shape, dtype, device, stream):
    """Memory of the stream that the call runs on: of another one's it could be in use still, or be used again too early."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


# A call's checks take as long as a small kernel does, so what is right is seen with few questions (each some 0.1 us), and what
# is wrong is asked again for its name.


def _current(t, what):
    """The device of a tensor, by number, which is the current one's."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError("%s must be a CUDA tensor" % what)
    device = t.get_device()
    if device != torch.cuda.current_device():
        raise ValueError("%s must be on the current device" % what)
    return device


def _refuse(t, what, dtype, device):
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError("%s must be a CUDA tensor" % what)
    if t.get_device() != device:
        raise ValueError("%s must be on device %d" % (what, device))
    if t.dtype != dtype:
        raise TypeError("%s must be of dtype %s" % (what, dtype))


def _flat(t, what, dtype, device, count):
    """Pointer of a contiguous tensor of `count` values."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.is_contiguous() and t.numel() == count):
        _refuse(t, what, dtype, device)
        if not t.is_contiguous():
            raise TypeError("%s must be contiguous" % what)
        raise ValueError("%s must hold %d values" % (what, count))
    return t.data_ptr()


# ---- residual join and norms ---------------------------------------------------------


class _Rows:
    """What the activations of a call have in common: shape, type, device, and the form that the library is given."""

    def __init__(self, like, kind, post, d_gate, residual_scale, eps):
        self.device = _current(like, "activations")
        self.dtype, self.shape = like.dtype, like.shape
        code = _DTYPES.get(self.dtype)
        if code is None or not self.shape:
            raise TypeError("activations must be float32, bfloat16 or float16 tensors of [..., cols]")
        self.cols = cols = self.shape[-1]
        self.form = Residual(like.numel() // cols if cols else 0, cols, code, kind, 1 if post else 0, ZT_GATE_NONE, residual_scale, eps)
        self.gate = None
        if d_gate is not None:
            if isinstance(d_gate, torch.Tensor) and d_gate.dim() == 1:
                self.form.gate, self.gate = ZT_GATE_CHANNEL, self.channels(d_gate, "d_gate")
            else:
                self.form.gate, self.gate = ZT_GATE_FULL, self.rows(d_gate, "gate")

    def rows(self, t, name):
        """Pointer of a tensor of the common shape and type whose rows are apart by one stride, which the form is told."""
        if isinstance(t, torch.Tensor) and t.is_contiguous() and t.dtype is self.dtype and t.get_device() == self.device and t.shape == self.shape:
            return t.data_ptr()      # stride 0 in the form: cols
        what = "d_" + name
        _refuse(t, what, self.dtype, self.device)
        if t.shape != self.shape:
            raise ValueError("%s must have shape %s" % (what, tuple(self.shape)))
        if t.dim() != 2:
            try:
                t = t.view(-1, self.cols)
            except RuntimeError:
                raise TypeError("%s: the distance from row to row must be the same everywhere" % what) from None
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise TypeError("%s: a row's values must lie next to one another" % what)
        if t.shape[0] > 1:
            if t.stride(0) == 0:
                raise TypeError("%s: rows that are all the same one (an expanded tensor) are not taken; make it contiguous" % what)
            setattr(self.form, "stride_" + name, t.stride(0))
        return t.data_ptr()

    def channels(self, t, what):
        return None if t is None else _flat(t, what, self.dtype, self.device, self.cols)

    def weights(self, post, pre_weight, pre_bias, post_weight, post_bias):
        if not post and (post_weight is not None or post_bias is not None):
            raise ValueError("post_weight and post_bias belong to a norm after the block: post=True")
        return (self.channels(pre_weight, "pre_weight"), self.channels(pre_bias, "pre_bias"), self.channels(post_weight, "post_weight"),
                self.channels(post_bias, "post_bias"))

    def empty(self, stream):
        return _empty(self.shape, self.dtype, self.device, stream)


def zt_residual_norm(d_x, d_b=None, kind=ZT_RMS, pre_weight=None, pre_bias=None, post=False, post_weight=None, post_bias=None, d_gate=None,
                     residual_scale=1.0, eps=1e-5, d_y=None, d_h=None, d_stats=None, stream=None, want_y=True):
    """y = residual_scale * d_x + gate * post(d_b), h = pre(y); returns (y, h).

    d_x and d_b are [..., cols]; d_gate is None, [cols] or of their shape.  d_stats, an fp32 tensor of rows x 4, gets what
    zt_residual_norm_backward needs.  want_y=False: y is not stored (and returned as None)."""
    r = _Rows(d_x, kind, post, d_gate, residual_scale, eps)
    weights = r.weights(post, pre_weight, pre_bias, post_weight, post_bias)
    if d_y is None and want_y:
        d_y = r.empty(stream)
    if d_h is None:
        d_h = r.empty(stream)
    x, b = r.rows(d_x, "x"), None if d_b is None else r.rows(d_b, "b")
    y, h = None if d_y is None else r.rows(d_y, "y"), r.rows(d_h, "h")
    stats = None if d_stats is None else _flat(d_stats, "d_stats", torch.float32, r.device, 4 * r.form.rows)
    _check(lib().zt_residual_norm(r.form, x, b, r.gate, *weights, y, h, stats, zc._stream_handle(stream)), "zt_residual_norm")
    return d_y, d_h


def zt_residual_norm_backward(d_dy, d_dh, d_y, d_b, d_stats, kind=ZT_RMS, pre_weight=None, pre_bias=None, post=False, post_weight=None,
                              post_bias=None, d_gate=None, residual_scale=1.0, d_dx=None, d_db=None, stream=None):
    """The gradients of zt_residual_norm from those of y (None for zero) and h, as a dict: "x", "b" and a full "gate" in the
    activations' type; "pre_weight", "pre_bias", "post_weight", "post_bias" and a channel "gate" in fp32; None for what the
    forward call did not have.  d_y is y as it was stored; the other arguments are the forward call's."""
    r = _Rows(d_dh, kind, post, d_gate, residual_scale, 0.0)
    pre_w, _, post_w, post_c = r.weights(post, pre_weight, pre_bias, post_weight, post_bias)
    if d_b is None and d_db is not None:
        raise ValueError("d_db without d_b")
    if d_dx is None:
        d_dx = r.empty(stream)
    if d_db is None and d_b is not None:
        d_db = r.empty(stream)
    full, channel = r.form.gate == ZT_GATE_FULL, r.form.gate == ZT_GATE_CHANNEL
    dgate = r.empty(stream) if full else None
    # the sums over the rows lie behind one another: a bucket of fp32 gradients
    wanted = (pre_weight is not None, pre_bias is not None, post_weight is not None, post_bias is not None, channel)
    sums = _empty((sum(wanted), r.cols), torch.float32, r.device, stream)
    at, pointers = sums.data_ptr(), []
    for w in wanted:
        pointers.append(at if w else None)
        at += 4 * r.cols if w else 0
    dh, y, dx = r.rows(d_dh, "dh"), r.rows(d_y, "y"), r.rows(d_dx, "dx")
    dy = None if d_dy is None else r.rows(d_dy, "dy")
    b, db = (None, None) if d_b is None else (r.rows(d_b, "b"), r.rows(d_db, "db"))
    stats = _flat(d_stats, "d_stats", torch.float32, r.device, 4 * r.form.rows)
    L = lib()
    size = L.zt_residual_work_bytes(r.form)
    work = _empty(size, torch.uint8, r.device, stream)
    _check(L.zt_residual_norm_backward(r.form, dy, dh, y, b, r.gate, pre_w, post_w, post_c, stats, dx, db, dgate.data_ptr() if full else pointers[4],
                                       *pointers[:4], work.data_ptr(), size, zc._stream_handle(stream)), "zt_residual_norm_backward")
    of = iter(sums.unbind(0))
    out = {"x": d_dx, "b": d_db}
    for name, w in zip(("pre_weight", "pre_bias", "post_weight", "post_bias", "gate"), wanted):
        out[name] = next(of) if w else None
    if full:
        out["gate"] = dgate
    return out


# ---- gradients -----------------------------------------------------------------------


_data_ptr, _numel, _get_device, _is_contiguous = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device, torch.Tensor.is_contiguous
_dtype = torch.Tensor.dtype.__get__     # as these, refuses what is no tensor with a TypeError


class _List:
    """Pointers, lengths and types of a list of tensors as C arrays."""

    def __init__(self, tensors, what):
        self.count = len(tensors)
        types = list(map(_DTYPES.get, map(_dtype, tensors)))
        self.device = torch.cuda.current_device() if tensors and None not in types and tensors[0].is_cuda else None
        if None in types or not all(map(_is_contiguous, tensors)) or (tensors and self.device is None):
            raise TypeError("%s must be contiguous CUDA tensors of dtype float32, bfloat16 or float16" % what)
        if tensors and set(map(_get_device, tensors)) != {self.device}:
            raise ValueError("%s must be on the current device" % what)
        self.pointers, self.lengths, self.types = array("Q", map(_data_ptr, tensors)), array("Q", map(_numel, tensors)), array("i", types)

    def arguments(self):
        return self.pointers.buffer_info()[0], self.lengths.buffer_info()[0], self.types.buffer_info()[0]


def _slots(d_slots):
    """Pointer and device of the partial sums of squares."""
    device = _current(d_slots, "d_slots")
    return _flat(d_slots, "d_slots", torch.float64, device, ZT_SLOTS), device


def _norm(d_norm, device, stream):
    """The tensor that gets the norm, and its pointer."""
    if d_norm is None:
        d_norm = _empty(1, torch.float32, device, stream)
        return d_norm, d_norm.data_ptr()
    return d_norm, _flat(d_norm, "d_norm", torch.float32, device, 1)


def zt_sum_squares(tensors, d_slots=None, accumulate=False, stream=None):
    """The sums of squares of a list of tensors as ZT_SLOTS doubles that add up to it; with accumulate added to d_slots.  Ranks
    add theirs up (an all-reduce of d_slots) before the norm is taken."""
    if accumulate and d_slots is None:
        raise ValueError("accumulate needs d_slots")
    tensors = _List(list(tensors), "tensors")
    if d_slots is None:
        d_slots = _empty(ZT_SLOTS, torch.float64, "cuda" if tensors.device is None else tensors.device, stream)
        slots = d_slots.data_ptr()
    else:
        slots, _ = _slots(d_slots)
    _check(lib().zt_sum_squares(*tensors.arguments(), tensors.count, 1 if accumulate else 0, slots, zc._stream_handle(stream)), "zt_sum_squares")
    return d_slots


def zt_norm(d_slots, scale=1.0, d_norm=None, stream=None):
    """scale * sqrt(the sum of squares): a tensor of one fp32 value."""
    slots, device = _slots(d_slots)
    d_norm, norm = _norm(d_norm, device, stream)
    _check(lib().zt_norm(slots, scale, norm, zc._stream_handle(stream)), "zt_norm")
    return d_norm


def zt_clip(tensors, max_norm, scale=1.0, d_out=None, d_slots=None, d_norm=None, stream=None):
    """Multiplies every tensor by scale, and by max_norm / norm if the norm of them all times scale is greater; returns the norm.

    d_out is a list of as many tensors of the same lengths, of any of the types; None: in place.  d_slots is what
    zt_sum_squares gave for them, summed over the ranks that share them out; None: it is taken here."""
    tensors = _List(list(tensors), "tensors")
    outs = tensors
    if d_out is not None:
        outs = _List(list(d_out), "d_out")
        if outs.lengths != tensors.lengths:
            raise ValueError("d_out must be as many tensors of the same lengths")
    handle, device = zc._stream_handle(stream), "cuda" if tensors.device is None else tensors.device
    arguments = tensors.arguments()
    if d_slots is None:
        d_slots = _empty(ZT_SLOTS, torch.float64, device, stream)
        slots = d_slots.data_ptr()
        _check(lib().zt_sum_squares(*arguments, tensors.count, 0, slots, handle), "zt_sum_squares")
    else:
        slots, device = _slots(d_slots)
    d_norm, norm = _norm(d_norm, device, stream)
    _check(lib().zt_clip(*arguments, outs.pointers.buffer_info()[0], outs.types.buffer_info()[0], tensors.count, slots, scale, max_norm, norm, handle), "zt_clip")
    return d_norm


def zt_adamw(d_grad, d_param, d_m, d_v, lr, beta1, beta2, eps, weight_decay, step, d_half=None, d_slots=None, scale=1.0, max_norm=float("inf"),
             d_norm=None, stream=None, d_state=None):
    """One AdamW step on a shard, in place: d_param, d_m and d_v are fp32, d_grad any type, d_half (bfloat16 or float16) gets
    the new parameters.  With d_slots (zt_sum_squares) the gradients are clipped to max_norm and the norm is returned; a limit
    without them is refused, since the norm to hold against it is that of all gradients and not of this shard's.

    lr and step are the call's: captured in a graph, it takes that step again in each replay.  With d_state, a float64 tensor of 4
    values [steps taken, learning rate, 0, 0], they are None; the call counts the step on the GPU, and does not where it leaves it out."""
    if (lr is None) != (d_state is not None) or (step is None) != (d_state is not None):
        raise ValueError("lr and step, or d_state in their place")
    if d_slots is None and max_norm != float("inf"):
        raise ValueError("max_norm needs d_slots")
    device = _current(d_grad, "d_grad")
    n, code = d_grad.numel(), _DTYPES.get(d_grad.dtype)
    if code is None:
        raise TypeError("d_grad must be of dtype float32, bfloat16 or float16")
    grad = _flat(d_grad, "d_grad", d_grad.dtype, device, n)
    param = _flat(d_param, "d_param", torch.float32, device, n)
    m, v = _flat(d_m, "d_m", torch.float32, device, n), _flat(d_v, "d_v", torch.float32, device, n)
    half, half_code, slots, norm = None, 0, None, None
    if d_half is not None:
        half_code = _DTYPES.get(d_half.dtype, zc.ZC_F32) if isinstance(d_half, torch.Tensor) else zc.ZC_F32
        if half_code == zc.ZC_F32:
            raise TypeError("d_half must be of dtype bfloat16 or float16")
        half = _flat(d_half, "d_half", d_half.dtype, device, n)
    if d_slots is not None:
        slots = _flat(d_slots, "d_slots", torch.float64, device, ZT_SLOTS)
        d_norm, norm = _norm(d_norm, device, stream)
    elif d_norm is not None:
        raise ValueError("d_norm needs d_slots")
    if d_state is None:
        form = AdamwForm(n, code, half_code, step, lr, beta1, beta2, eps, weight_decay, scale, max_norm, None)
    else:
        form = AdamwForm(n, code, half_code, 0, 0.0, beta1, beta2, eps, weight_decay, scale, max_norm, _flat(d_state, "d_state", torch.float64, device, 4))
    _check(lib().zt_adamw(form, grad, slots, param, m, v, half, norm, zc._stream_handle(stream)), "zt_adamw")
    return d_norm
