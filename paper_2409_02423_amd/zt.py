"""Python binding of the training-step operators of libzc (include/zt.h): argument marshalling only.

Every function has the name and meaning of the C entry point it calls.  Tensors are torch CUDA tensors of the
current device, used as device memory; the kernels are enqueued on torch's current stream unless a stream is given, and what a
call allocates (outputs that are not passed, workspaces) belongs to the stream it runs on.  There is no fallback: if the HIP
library cannot be loaded, every call raises.
"""
import ctypes

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
                ("weight_decay", ctypes.c_double), ("scale", ctypes.c_float), ("max_norm", ctypes.c_float)]


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


def _on_device(t, what, device=None):
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError("%s must be a CUDA tensor" % what)
    if t.device.index != torch.cuda.current_device() if device is None else t.device != device:
        raise ValueError("%s must be on %s" % (what, "the current device" if device is None else device))


def _flat(t, what, dtype=None, device=None):
    """A contiguous tensor's pointer."""
    _on_device(t, what, device)
    if not t.is_contiguous() or (t.dtype not in _DTYPES if dtype is None else t.dtype != dtype):
        raise TypeError("%s must be contiguous, of dtype %s" % (what, dtype or "float32, bfloat16 or float16"))
    return t.data_ptr()


# ---- residual join and norms ---------------------------------------------------------


def _rows_of(t, like, what):
    """Pointer of a tensor of like's shape and type whose rows are apart by one stride, and that stride."""
    _on_device(t, what, like.device)
    if t.dtype != like.dtype:
        raise TypeError("%s must be of dtype %s" % (what, like.dtype))
    if t.shape != like.shape:
        raise ValueError("%s must have shape %s" % (what, tuple(like.shape)))
    if t.is_contiguous():
        return t.data_ptr(), like.shape[-1]
    if t.dim() != 2:
        try:
            t = t.view(-1, t.shape[-1])
        except RuntimeError:
            raise TypeError("%s: the distance from row to row must be the same everywhere" % what) from None
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise TypeError("%s: a row's values must lie next to one another" % what)
    if t.shape[0] > 1 and t.stride(0) == 0:
        raise TypeError("%s: rows that are all the same one (an expanded tensor) are not taken; make it contiguous" % what)
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else like.shape[-1]


def _channels(t, like, what):
    if t is None:
        return None
    pointer = _flat(t, what, like.dtype, like.device)
    if t.numel() != like.shape[-1]:
        raise ValueError("%s must hold %d values" % (what, like.shape[-1]))
    return pointer


def _form(like, kind, post, d_gate, residual_scale, eps):
    if not (isinstance(like, torch.Tensor) and like.is_cuda):
        raise TypeError("activations must be CUDA tensors")
    _on_device(like, "activations")
    if like.dtype not in _DTYPES or like.dim() == 0:
        raise TypeError("activations must be float32, bfloat16 or float16 tensors of [..., cols]")
    cols = like.shape[-1]
    f = Residual(rows=like.numel() // cols if cols else 0, cols=cols, dtype=_DTYPES[like.dtype], kind=kind, post=1 if post else 0,
                 residual_scale=residual_scale, eps=eps)
    gate = None
    if d_gate is not None:
        if d_gate.dim() == 1:
            f.gate, gate = ZT_GATE_CHANNEL, _channels(d_gate, like, "d_gate")
        else:
            f.gate = ZT_GATE_FULL
            gate, f.stride_gate = _rows_of(d_gate, like, "d_gate")
    return f, gate


def _without_post(post, post_weight, post_bias):
    if not post and (post_weight is not None or post_bias is not None):
        raise ValueError("post_weight and post_bias belong to a norm after the block: post=True")


def zt_residual_norm(d_x, d_b=None, kind=ZT_RMS, pre_weight=None, pre_bias=None, post=False, post_weight=None, post_bias=None, d_gate=None,
                     residual_scale=1.0, eps=1e-5, d_y=None, d_h=None, d_stats=None, stream=None, want_y=True):
    """y = residual_scale * d_x + gate * post(d_b), h = pre(y); returns (y, h).

    d_x and d_b are [..., cols]; d_gate is None, [cols] or of their shape.  d_stats, an fp32 tensor of rows x 4, gets what
    zt_residual_norm_backward needs.  want_y=False: y is not stored (and returned as None)."""
    f, gate = _form(d_x, kind, post, d_gate, residual_scale, eps)
    _without_post(post, post_weight, post_bias)
    x, f.stride_x = _rows_of(d_x, d_x, "d_x")
    b = y = None
    if d_b is not None:
        b, f.stride_b = _rows_of(d_b, d_x, "d_b")
    if d_y is None and want_y:
        d_y = _empty(d_x.shape, d_x.dtype, d_x.device, stream)
    if d_y is not None:
        y, f.stride_y = _rows_of(d_y, d_x, "d_y")
    if d_h is None:
        d_h = _empty(d_x.shape, d_x.dtype, d_x.device, stream)
    h, f.stride_h = _rows_of(d_h, d_x, "d_h")
    stats = None
    if d_stats is not None:
        stats = _flat(d_stats, "d_stats", torch.float32, d_x.device)
        if d_stats.numel() != 4 * f.rows:
            raise ValueError("d_stats must hold four floats for each of the %d rows" % f.rows)
    _check(lib().zt_residual_norm(f, x, b, gate, _channels(pre_weight, d_x, "pre_weight"), _channels(pre_bias, d_x, "pre_bias"),
                                  _channels(post_weight, d_x, "post_weight"), _channels(post_bias, d_x, "post_bias"), y, h, stats,
                                  zc._stream_handle(stream)), "zt_residual_norm")
    return d_y, d_h


def zt_residual_norm_backward(d_dy, d_dh, d_y, d_b, d_stats, kind=ZT_RMS, pre_weight=None, pre_bias=None, post=False, post_weight=None,
                              post_bias=None, d_gate=None, residual_scale=1.0, d_dx=None, d_db=None, stream=None):
    """The gradients of zt_residual_norm from those of y (None for zero) and h, as a dict: "x", "b" and a full "gate" in the
    activations' type; "pre_weight", "pre_bias", "post_weight", "post_bias" and a channel "gate" in fp32; None for what the
    forward call did not have.  d_y is y as it was stored; the other arguments are the forward call's."""
    f, gate = _form(d_dh, kind, post, d_gate, residual_scale, 0.0)
    _without_post(post, post_weight, post_bias)
    device, cols = d_dh.device, d_dh.shape[-1]
    dh, f.stride_dh = _rows_of(d_dh, d_dh, "d_dh")
    y, f.stride_y = _rows_of(d_y, d_dh, "d_y")
    dy = b = db = None
    if d_dy is not None:
        dy, f.stride_dy = _rows_of(d_dy, d_dh, "d_dy")
    if d_dx is None:
        d_dx = _empty(d_dh.shape, d_dh.dtype, device, stream)
    dx, f.stride_dx = _rows_of(d_dx, d_dh, "d_dx")
    if d_b is not None:
        b, f.stride_b = _rows_of(d_b, d_dh, "d_b")
        if d_db is None:
            d_db = _empty(d_dh.shape, d_dh.dtype, device, stream)
        db, f.stride_db = _rows_of(d_db, d_dh, "d_db")
    elif d_db is not None:
        raise ValueError("d_db without d_b")
    stats = _flat(d_stats, "d_stats", torch.float32, device)
    if d_stats.numel() != 4 * f.rows:
        raise ValueError("d_stats must hold four floats for each of the %d rows" % f.rows)
    pre_w, post_w, post_c = _channels(pre_weight, d_dh, "pre_weight"), _channels(post_weight, d_dh, "post_weight"), _channels(post_bias, d_dh, "post_bias")
    _channels(pre_bias, d_dh, "pre_bias")
    out = {"x": d_dx, "b": d_db, "gate": None}
    if f.gate == ZT_GATE_FULL:
        out["gate"] = _empty(d_dh.shape, d_dh.dtype, device, stream)
    # the sums over the rows, one allocation for all: it is a bucket of fp32 gradients
    names = [n for n, t in (("pre_weight", pre_weight), ("pre_bias", pre_bias), ("post_weight", post_weight), ("post_bias", post_bias)) if t is not None]
    if f.gate == ZT_GATE_CHANNEL:
        names.append("gate")
    sums = _empty((len(names), cols), torch.float32, device, stream)
    for n in ("pre_weight", "pre_bias", "post_weight", "post_bias"):
        out[n] = None
    for i, n in enumerate(names):
        out[n] = sums[i]
    work = _empty(int(lib().zt_residual_work_bytes(f)), torch.uint8, device, stream)

    def pointer(name):
        return None if out[name] is None else out[name].data_ptr()

    _check(lib().zt_residual_norm_backward(f, dy, dh, y, b, gate, pre_w, post_w, post_c, stats, dx, db, pointer("gate"), pointer("pre_weight"),
                                           pointer("pre_bias"), pointer("post_weight"), pointer("post_bias"), work.data_ptr(), work.numel(),
                                           zc._stream_handle(stream)), "zt_residual_norm_backward")
    return out


# ---- gradients -----------------------------------------------------------------------


def _list(tensors, what):
    """Pointers, lengths and types of a list of tensors as C arrays."""
    count = len(tensors)
    pointers, lengths, types = (ctypes.c_void_p * max(count, 1))(), (ctypes.c_size_t * max(count, 1))(), (ctypes.c_int * max(count, 1))()
    device = None
    for i, t in enumerate(tensors):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in _DTYPES and t.is_contiguous()):
            raise TypeError("%s must be contiguous CUDA tensors of dtype float32, bfloat16 or float16" % what)
        if device is None:
            device = torch.cuda.current_device()
        if t.get_device() != device:
            raise ValueError("%s must be on the current device" % what)
        pointers[i], lengths[i], types[i] = t.data_ptr(), t.numel(), _DTYPES[t.dtype]
    return pointers, lengths, types, count


def _check_slots(d_slots):
    pointer = _flat(d_slots, "d_slots", torch.float64)
    if d_slots.numel() != ZT_SLOTS:
        raise ValueError("d_slots must hold %d values" % ZT_SLOTS)
    return pointer


def _check_norm(d_norm):
    pointer = _flat(d_norm, "d_norm", torch.float32)
    if d_norm.numel() < 1:
        raise ValueError("d_norm must hold a value")
    return pointer


def zt_sum_squares(tensors, d_slots=None, accumulate=False, stream=None):
    """The sums of squares of a list of tensors as ZT_SLOTS doubles that add up to it; with accumulate added to d_slots.  Ranks
    add theirs up (an all-reduce of d_slots) before the norm is taken."""
    if accumulate and d_slots is None:
        raise ValueError("accumulate needs d_slots")
    pointers, lengths, types, count = _list(list(tensors), "tensors")
    if d_slots is None:
        d_slots = _empty(ZT_SLOTS, torch.float64, "cuda", stream)
    _check(lib().zt_sum_squares(pointers, lengths, types, count, 1 if accumulate else 0, _check_slots(d_slots), zc._stream_handle(stream)), "zt_sum_squares")
    return d_slots


def zt_norm(d_slots, scale=1.0, d_norm=None, stream=None):
    """scale * sqrt(the sum of squares): a tensor of one fp32 value."""
    slots = _check_slots(d_slots)
    if d_norm is None:
        d_norm = _empty(1, torch.float32, d_slots.device, stream)
    _check(lib().zt_norm(slots, scale, _check_norm(d_norm), zc._stream_handle(stream)), "zt_norm")
    return d_norm


def zt_clip(tensors, max_norm, scale=1.0, d_out=None, d_slots=None, d_norm=None, stream=None):
    """Multiplies every tensor by scale, and by max_norm / norm if the norm of them all times scale is greater; returns the norm.

    d_out is a list of as many tensors of the same lengths, of any of the types; None: in place.  d_slots is what
    zt_sum_squares gave for them, summed over the ranks that share them out; None: it is taken here."""
    tensors = list(tensors)
    pointers, lengths, types, count = _list(tensors, "tensors")
    if d_out is None:
        outs, out_types = pointers, types
    else:
        d_out = list(d_out)
        outs, out_lengths, out_types, out_count = _list(d_out, "d_out")
        if out_count != count or list(out_lengths) != list(lengths):
            raise ValueError("d_out must be as many tensors of the same lengths")
    handle = zc._stream_handle(stream)
    if d_slots is None:
        d_slots = _empty(ZT_SLOTS, torch.float64, "cuda", stream)
        slots = d_slots.data_ptr()
        _check(lib().zt_sum_squares(pointers, lengths, types, count, 0, slots, handle), "zt_sum_squares")
    else:
        slots = _check_slots(d_slots)
    if d_norm is None:
        d_norm = _empty(1, torch.float32, "cuda", stream)
    _check(lib().zt_clip(pointers, lengths, types, outs, out_types, count, slots, scale, max_norm, _check_norm(d_norm), handle), "zt_clip")
    return d_norm


def zt_adamw(d_grad, d_param, d_m, d_v, lr, beta1, beta2, eps, weight_decay, step, d_half=None, d_slots=None, scale=1.0, max_norm=float("inf"),
             d_norm=None, stream=None):
    """One AdamW step on a shard, in place: d_param, d_m and d_v are fp32, d_grad any type, d_half (bfloat16 or float16) gets
    the new parameters.  With d_slots (zt_sum_squares) the gradients are clipped to max_norm and the norm is returned."""
    grad = _flat(d_grad, "d_grad")
    form = AdamwForm(n=d_grad.numel(), grad_dtype=_DTYPES[d_grad.dtype], step=step, lr=lr, beta1=beta1, beta2=beta2, eps=eps,
                     weight_decay=weight_decay, scale=scale, max_norm=max_norm)
    pointers = []
    for t, what in ((d_param, "d_param"), (d_m, "d_m"), (d_v, "d_v")):
        pointers.append(_flat(t, what, torch.float32))
        if t.numel() != form.n:
            raise ValueError("%s must hold %d values" % (what, form.n))
    half = slots = norm = None
    if d_half is not None:
        half = _flat(d_half, "d_half")
        if d_half.numel() != form.n:
            raise ValueError("d_half must hold %d values" % form.n)
        form.half_dtype = _DTYPES[d_half.dtype]
    if d_slots is not None:
        slots = _check_slots(d_slots)
        if d_norm is None:
            d_norm = _empty(1, torch.float32, d_grad.device, stream)
    elif d_norm is not None:
        raise ValueError("d_norm needs d_slots")
    if d_norm is not None:
        norm = _check_norm(d_norm)
    _check(lib().zt_adamw(form, grad, slots, *pointers, half, norm, zc._stream_handle(stream)), "zt_adamw")
    return d_norm
