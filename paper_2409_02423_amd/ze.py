"""Python binding of the vocabulary's operators of libzc (include/ze.h): argument marshalling only.

Every function has the name and meaning of the C entry point it calls.  Tensors are torch CUDA tensors of the
current device, used as device memory; the kernels are enqueued on torch's current stream unless a stream is given, and what a
call allocates (outputs that are not passed, workspaces) belongs to the stream it runs on.  There is no fallback: if the HIP
library cannot be loaded, every call raises.
"""
import ctypes

import torch

from . import zc
from .zc import ZC_OK, ZcError  # noqa: F401
from .zt import ZC_ERR_ARG, _check, _current, _DTYPES, _empty, _flat, _refuse  # noqa: F401

ZE_I32, ZE_I64 = 0, 1
ZE_MAX_TOKENS, ZE_MAX_ROWS, ZE_MAX_COLS = 1 << 25, 1 << 28, 65536
_MOST_FIRST = (1 << 63) - 1 - ZE_MAX_ROWS

EXPORTS = ("ze_embedding", "ze_embedding_work_bytes", "ze_embedding_backward", "ze_loss_work_bytes", "ze_vocab_loss", "ze_join_loss",
           "ze_loss_backward_work_bytes", "ze_vocab_loss_backward")

_IDS = {torch.int32: ZE_I32, torch.int64: ZE_I64}


class Form(ctypes.Structure):
    """struct ze_form"""
    _fields_ = [("tokens", ctypes.c_size_t), ("rows", ctypes.c_size_t), ("cols", ctypes.c_size_t), ("first", ctypes.c_longlong), ("dtype", ctypes.c_int),
                ("grad_dtype", ctypes.c_int), ("id_dtype", ctypes.c_int), ("scale", ctypes.c_float)] + [
                    ("stride_" + name, ctypes.c_size_t) for name in ("table", "tokens", "dtable", "dtokens")]


_lib = None


def lib():
    """The loaded C library (zc.lib()) with these operators' signatures."""
    global _lib
    L = zc.lib()
    if _lib is not L:
        p, size, form = ctypes.c_void_p, ctypes.c_size_t, ctypes.POINTER(Form)
        L.ze_embedding.argtypes = [form, p, p, p, p]
        L.ze_embedding_work_bytes.restype = size
        L.ze_embedding_work_bytes.argtypes = [form]
        L.ze_embedding_backward.argtypes = [form, p, p, p, ctypes.c_int, p, size, p]
        L.ze_loss_work_bytes.restype = size
        L.ze_loss_work_bytes.argtypes = [form, p, p]
        L.ze_vocab_loss.argtypes = [form, p, p, p, p, p, size, p]
        L.ze_join_loss.argtypes = [size, ctypes.c_int, ctypes.c_int, p, p, p, p, p]
        L.ze_loss_backward_work_bytes.restype = size
        L.ze_loss_backward_work_bytes.argtypes = [form, p, p, size]
        L.ze_vocab_loss_backward.argtypes = [form, p, p, p, p, p, p, p, size, p, size, p]
        _lib = L
    return _lib


# A call's checks take as long as a small kernel does, so what is right is seen with few questions, and what is wrong is asked again for its name.


class _Call:
    """What the tensors of a call have in common, and the form that the library is given."""
    __slots__ = ("device", "dtype", "shape", "table_shape", "tokens_shape", "ids", "form")

    def __init__(self, d_ids, what, like, like_what, rows, first, scale):
        # (what does not fit into the form's fields would be cut to their width, without an error)
        if not 0 <= first <= _MOST_FIRST:
            raise ZcError(ZC_ERR_ARG, "first = %d" % first)
        if not 0 <= rows <= ZE_MAX_ROWS:
            raise ZcError(zc.ZC_ERR_SIZE, "rows = %d" % rows)
        device = self.device = _current(like, like_what)
        dtype = self.dtype = like.dtype
        code, of = _DTYPES.get(dtype), like.shape
        if code is None or not of:
            raise TypeError("%s must be a float32, bfloat16 or float16 tensor of [..., cols]" % like_what)
        cols = of[-1]
        ids = _IDS.get(d_ids.dtype) if isinstance(d_ids, torch.Tensor) else None
        if ids is None:
            raise TypeError("%s must be a CUDA tensor of dtype int32 or int64" % what)
        count = d_ids.numel()
        if not (d_ids.get_device() == device and d_ids.is_contiguous()):
            _flat(d_ids, what, d_ids.dtype, device, count)
        self.ids = d_ids.data_ptr()
        shape = self.shape = d_ids.shape
        self.table_shape, self.tokens_shape = (rows, cols), (count, cols) if len(shape) == 1 else (*shape, cols)
        self.form = Form(count, rows, cols, first, code, code, ids, scale)

    def table(self, t, what, name, dtype=None):
        """Pointer of a [rows, cols] tensor whose rows are apart by a stride, which the form is told."""
        dtype = dtype or self.dtype
        if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == self.device and t.is_contiguous() and t.shape == self.table_shape:
            return t.data_ptr()      # stride 0 in the form: cols
        _refuse(t, what, dtype, self.device)
        if t.shape != self.table_shape:
            raise ValueError("%s must have shape %s" % (what, self.table_shape))
        return self._rows(t, what, name)

    def tokens(self, t, what, name):
        """Pointer of a tensor with a row for each id."""
        if isinstance(t, torch.Tensor) and t.dtype is self.dtype and t.get_device() == self.device and t.is_contiguous() and t.shape == self.tokens_shape:
            return t.data_ptr()
        _refuse(t, what, self.dtype, self.device)
        if t.shape != self.tokens_shape:
            raise ValueError("%s must have shape %s" % (what, self.tokens_shape))
        if t.dim() != 2:
            try:
                t = t.view(-1, self.form.cols)
            except RuntimeError:
                raise TypeError("%s: the distance from row to row must be the same everywhere" % what) from None
        return self._rows(t, what, name)

    def _rows(self, t, what, name):
        if t.is_contiguous():
            return t.data_ptr()
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise TypeError("%s: a row's values must lie next to one another" % what)
        if t.shape[0] > 1:
            if t.stride(0) == 0:
                raise TypeError("%s: rows that are all the same one (an expanded tensor) are not taken; make it contiguous" % what)
            setattr(self.form, "stride_" + name, t.stride(0))
        return t.data_ptr()

    def floats(self, t, what, count=None):
        return _flat(t, what, torch.float32, self.device, self.form.tokens if count is None else count)

    def empty(self, shape, dtype, stream):
        return _empty(shape, dtype, self.device, stream)

    def work(self, size, stream):
        """Workspace of a call, and its pointer."""
        if not size:
            return None, None
        work = _empty(size, torch.uint8, self.device, stream)
        return work, work.data_ptr()


def _rows_of(d_table):
    return d_table.shape[0] if isinstance(d_table, torch.Tensor) and d_table.dim() else 0


# ---- embedding -----------------------------------------------------------------------


def ze_embedding(d_ids, d_table, first=0, scale=1.0, d_out=None, stream=None):
    """scale * d_table[id - first] for each id, zeros for ids that are not this rank's; returns d_out, [..., cols] for ids of [...]."""
    c = _Call(d_ids, "d_ids", d_table, "d_table", _rows_of(d_table), first, scale)
    table = c.table(d_table, "d_table", "table")
    if d_out is None:
        d_out = c.empty(c.tokens_shape, c.dtype, stream)
    out = c.tokens(d_out, "d_out", "dtokens")
    rc = lib().ze_embedding(c.form, c.ids, table, out, zc._stream_handle(stream))
    if rc:
        _check(rc, "ze_embedding")
    return d_out


def ze_embedding_backward(d_ids, d_dout, rows, first=0, scale=1.0, d_dtable=None, accumulate=False, stream=None):
    """The gradient of the table's `rows` rows from that of the lookup's output: scale times the sum over each row's tokens, in fp32 or, as d_dtable
    is, in d_dout's type.  With accumulate it is added to what d_dtable holds."""
    if accumulate and d_dtable is None:
        raise ValueError("accumulate needs d_dtable")
    c = _Call(d_ids, "d_ids", d_dout, "d_dout", rows, first, scale)
    dout = c.tokens(d_dout, "d_dout", "tokens")
    if d_dtable is None:
        d_dtable = c.empty(c.table_shape, torch.float32, stream)
    dtype = c.dtype if isinstance(d_dtable, torch.Tensor) and d_dtable.dtype is c.dtype else torch.float32
    dtable = c.table(d_dtable, "d_dtable", "dtable", dtype)
    c.form.grad_dtype = _DTYPES[dtype]
    L = lib()
    size = L.ze_embedding_work_bytes(c.form)
    work, at = c.work(size, stream)
    _check(L.ze_embedding_backward(c.form, c.ids, dout, dtable, 1 if accumulate else 0, at, size, zc._stream_handle(stream)), "ze_embedding_backward")
    return d_dtable


# ---- softmax cross entropy -----------------------------------------------------------


def _loss_call(d_hidden, d_table, d_labels, first, scale):
    c = _Call(d_labels, "d_labels", d_hidden, "d_hidden", _rows_of(d_table), first, scale)
    return c, c.tokens(d_hidden, "d_hidden", "tokens"), c.table(d_table, "d_table", "table")


def ze_vocab_loss(d_hidden, d_table, d_labels, first=0, scale=1.0, d_stats=None, stream=None):
    """This rank's part of the softmax cross entropy of d_hidden [..., cols] against its rows d_table [rows, cols], as d_stats [3, tokens]: for each
    token the greatest logit, the sum of exponentials, the label's logit.  A negative label leaves its token out."""
    c, hidden, table = _loss_call(d_hidden, d_table, d_labels, first, scale)
    if d_stats is None:
        d_stats = c.empty((3, c.form.tokens), torch.float32, stream)
    stats = c.floats(d_stats, "d_stats", 3 * c.form.tokens)
    L = lib()
    size = L.ze_loss_work_bytes(c.form, hidden, table)
    work, at = c.work(size, stream)
    _check(L.ze_vocab_loss(c.form, hidden, table, c.ids, stats, at, size, zc._stream_handle(stream)), "ze_vocab_loss")
    return d_stats


def ze_join_loss(d_stats, d_labels, d_loss=None, d_lse=None, stream=None):
    """(loss, lse) of each token, in the labels' shape, from the d_stats of all ranks, [ranks, 3, tokens] (or one rank's, [3, tokens])."""
    device = _current(d_stats, "d_stats")
    ids = _IDS.get(d_labels.dtype) if isinstance(d_labels, torch.Tensor) else None
    if ids is None:
        raise TypeError("d_labels must be a CUDA tensor of dtype int32 or int64")
    tokens = d_labels.numel()
    if d_stats.dim() not in (2, 3) or d_stats.shape[-2] != 3 or d_stats.shape[-1] != tokens:
        raise ValueError("d_stats must have shape (ranks, 3, %d)" % tokens)
    ranks = d_stats.shape[0] if d_stats.dim() == 3 else 1
    labels = _flat(d_labels, "d_labels", d_labels.dtype, device, tokens)
    stats = _flat(d_stats, "d_stats", torch.float32, device, ranks * 3 * tokens)
    if d_loss is None:
        d_loss = _empty(d_labels.shape, torch.float32, device, stream)
    if d_lse is None:
        d_lse = _empty(d_labels.shape, torch.float32, device, stream)
    loss, lse = _flat(d_loss, "d_loss", torch.float32, device, tokens), _flat(d_lse, "d_lse", torch.float32, device, tokens)
    _check(lib().ze_join_loss(tokens, ranks, ids, stats, labels, loss, lse, zc._stream_handle(stream)), "ze_join_loss")
    return d_loss, d_lse


def ze_vocab_loss_backward(d_hidden, d_table, d_labels, d_lse, d_dloss, first=0, scale=1.0, d_dhidden=None, d_dtable=None, stream=None, want_hidden=True,
                           want_table=True, piece=0):
    """(d_dhidden, d_dtable): the gradients of the hidden states (this rank's part, to be added up over the ranks) and of this rank's rows, from d_lse
    (ze_join_loss) and the gradient of each token's loss.  want_hidden or want_table False: that one is not computed (and None).
    piece: rows of the table whose probabilities lie in the workspace at a time, 0 for the library's choice.  d_dhidden may be d_hidden."""
    c, hidden, table = _loss_call(d_hidden, d_table, d_labels, first, scale)
    if (d_dhidden is not None and not want_hidden) or (d_dtable is not None and not want_table):
        raise ValueError("an output that is not wanted")
    if piece < 0:
        raise ValueError("piece must not be negative")
    if d_dhidden is None and want_hidden:
        d_dhidden = c.empty(d_hidden.shape, c.dtype, stream)
    if d_dtable is None and want_table:
        d_dtable = c.empty(d_table.shape, c.dtype, stream)
    dhidden = c.tokens(d_dhidden, "d_dhidden", "dtokens") if want_hidden else None
    dtable = c.table(d_dtable, "d_dtable", "dtable") if want_table else None
    lse, dloss = c.floats(d_lse, "d_lse"), c.floats(d_dloss, "d_dloss")
    piece = min(piece, ZE_MAX_ROWS)      # (as many rows as there can be; more would be cut to the argument's width)
    L = lib()
    size = L.ze_loss_backward_work_bytes(c.form, hidden, table, piece)
    work, at = c.work(size, stream)
    _check(L.ze_vocab_loss_backward(c.form, hidden, table, c.ids, lse, dloss, dhidden, dtable, piece, at, size, zc._stream_handle(stream)), "ze_vocab_loss_backward")
    return d_dhidden, d_dtable
