"""Operators of a head that is trained on a topic model's features and answers from them, on torch tensors in device memory.

``layer_norm``, ``rms_norm``, ``linear_cross_entropy``   differentiable, for a training loop written with torch
``layer_norm_forward`` / ``_backward``, ``rms_norm_forward`` / ``_backward``, ``linear_cross_entropy_forward`` / ``_backward``   the
                                           passes themselves
``checkpoint8``                            an activation held in 8 bits
``rms_norm8``, ``rows8``, ``linear8``      serving in 8 bits: the norm's output, rows of a matrix, logits from both
``sample``                                 a word drawn for every row of logits: temperature, top-k, top-p, min-p

The work is done by the HIP kernels behind the C ABI of ``include/saber_ops.h``; torch supplies memory, streams and
the graph of gradients.  Everything is enqueued on torch's current stream of the tensors' device: nothing is waited
for, and calls may be captured into a graph (a backward pass by autograd as any of torch's: while no graph of gradients
that was made outside of the capture is alive on the same leaves; the passes themselves always).  Arguments are checked on the host (ValueError, TypeError, or SaberError
from the library).  There is no CPU fallback.

A program that uses the sampler as well imports torch before it: the library then runs on torch's HIP runtime.  Loaded
first it brings the system's, which knows neither torch's streams nor the order of its work, and importing this module
raises ImportError.
"""
from __future__ import annotations

import ctypes
import operator
import os

import torch
from torch.autograd import forward_ad

from ..binding import SABER_OK, SaberError, load_library

__all__ = ["Checkpoint8", "NormSaved", "RmsSaved", "Rows8", "checkpoint8", "layer_norm", "layer_norm_backward", "layer_norm_forward", "linear8",
           "linear_cross_entropy", "linear_cross_entropy_backward", "linear_cross_entropy_forward", "rms_norm", "rms_norm8",
           "rms_norm_backward", "rms_norm_forward", "rows8", "sample"]

BLOCK = 128   # columns that share a step of a checkpoint

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_int64 = ctypes.c_int64
_F32 = torch.float32

_L = load_library()


def _check_runtime():
    """That the library and torch share one HIP runtime: a second one in the process is the one the library was loaded with."""
    with open("/proc/self/maps") as f:
        paths = {os.path.realpath(line.split(None, 5)[5].strip()) for line in f if "/libamdhip64" in line}
    if len(paths) > 1:
        raise ImportError("libsaber.so was loaded before torch, on another HIP runtime than torch's (%s): import torch before the "
                          "first use of paper_1610_02496_amd" % ", ".join(sorted(paths)))


_check_runtime()
_norm_forward, _norm_backward, _norm_space = (_L.saber_layer_norm_forward, _L.saber_layer_norm_backward,
                                              _L.saber_layer_norm_backward_workspace)
_save8, _restore8 = _L.saber_checkpoint8_save, _L.saber_checkpoint8_restore
_xent_forward, _xent_backward = _L.saber_linear_xent_forward, _L.saber_linear_xent_backward
_rms_forward, _rms_backward, _rms_space = _L.saber_rms_norm_forward, _L.saber_rms_norm_backward, _L.saber_rms_norm_backward_workspace
_rows8_save, _rows8_restore, _linear8, _sample = _L.saber_rows8_save, _L.saber_rows8_restore, _L.saber_linear8, _L.saber_sample

# without the objects that torch.cuda.current_stream() makes on every call (2 us of a call of 12)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(call, device, *args):
    """The call on the current stream of the tensors' device."""
    index = device.index
    if _current_device() == index:
        rc = call(*args, _current_stream(index))
    else:
        with torch.cuda.device(index):
            rc = call(*args, _current_stream(index))
    if rc != SABER_OK:
        _check(rc)


def _check(rc):
    if rc != SABER_OK:
        raise SaberError(rc, _L.saber_ops_last_error().decode("utf-8", "replace"))


def _type(name, t):
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError("%s must be float32, float16 or bfloat16, not %s" % (name, t.dtype))
    return code


def _device(t, name, like=None):
    """The device of a tensor in device memory: that of `like` where there is one."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be in device memory, not on %s" % (name, t.device))
    if like is not None and t.device != like:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, like))
    return t.device


def _rows(t, name):
    """(matrix, rows, columns, elements between rows) of a tensor seen as a matrix of its last dimension, without a copy where
    the layout allows it; the matrix is the tensor itself, or a contiguous copy."""
    shape = t.shape
    if len(shape) == 2:
        rows, cols = shape
        stride, one = t.stride()
        if (one == 1 or cols == 1) and (stride >= cols or rows <= 1):
            return t, rows, cols, stride if stride >= cols else cols
        return t.contiguous(), rows, cols, cols
    if not shape:
        raise ValueError("%s has no columns" % name)
    cols = shape[-1]
    return t.contiguous(), t.numel() // cols if cols else 0, cols, cols


def _vector(t, name, cols, like, of):
    _device(t, name, like)
    if t.shape != (cols,):
        raise ValueError("%s must hold %d values, one per column of %s" % (name, cols, of))
    return t if t.is_contiguous() else t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---- checkpoints in 8 bits -------------------------------------------------------------------------------------------

class Checkpoint8:
    """An activation in 8 bits: ``q`` (int8, the shape of the activation) times ``scale`` (float32, one step per 128
    columns of a row).  An element is off by half a step at most, a 254th of its block's largest magnitude (blocks whose
    largest is below 2^-119, where steps are not normal numbers, are held more coarsely)."""

    __slots__ = ("q", "scale", "dtype")

    def __init__(self, q, scale, dtype):
        self.q, self.scale, self.dtype = q, scale, dtype

    def restore(self, dtype=None):
        """The activation, in its own type or another floating type."""
        q = self.q
        x = torch.empty_like(q, dtype=dtype or self.dtype)
        cols = q.shape[-1]
        _launch(_restore8, q.device, q.data_ptr(), self.scale.data_ptr(), q.numel() // cols if cols else 0, cols, _type("dtype", x), x.data_ptr())
        return x


def _empty_checkpoint(x, rows, cols):
    return Checkpoint8(x.new_empty(x.shape, dtype=torch.int8), x.new_empty((rows, (cols + BLOCK - 1) // BLOCK), dtype=_F32), x.dtype)


def checkpoint8(x) -> Checkpoint8:
    """Holds ``x`` (any shape, blocks run along its last dimension) in 8 bits."""
    device = _device(x, "x")
    code = _type("x", x)
    m, rows, cols, stride = _rows(x, "x")
    c = _empty_checkpoint(x, rows, cols)
    _launch(_save8, device, m.data_ptr(), stride, rows, cols, code, c.q.data_ptr(), c.scale.data_ptr())
    return c


# ---- layer norm ------------------------------------------------------------------------------------------------------

class NormSaved:
    """What the backward pass of a layer norm needs: its input (or an 8-bit checkpoint of it), its weight, and mean and
    1 / standard deviation of every row."""

    __slots__ = ("x", "checkpoint", "weight", "bias", "mean", "rstd")

    def __init__(self, x, checkpoint, weight, bias, mean, rstd):
        self.x, self.checkpoint, self.weight, self.bias, self.mean, self.rstd = x, checkpoint, weight, bias, mean, rstd


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, checkpoint=False):
    """Layer norm over the last dimension: ``(y, saved)``.  ``weight`` and ``bias`` are vectors of one floating type (their
    own or that of ``x``).  With ``checkpoint`` the input is held in 8 bits for the backward pass, written in the same
    pass over ``x``; ``x`` itself is not kept."""
    device = _device(x, "x")
    code = wcode = _type("x", x)
    m, rows, cols, stride = _rows(x, "x")
    if weight is not None:
        weight = _vector(weight, "weight", cols, device, "x")
        wcode = _type("weight", weight)
    if bias is not None:
        bias = _vector(bias, "bias", cols, device, "x")
        if weight is None:
            wcode = _type("bias", bias)
        elif bias.dtype != weight.dtype:
            raise TypeError("weight and bias must have one type, not %s and %s" % (weight.dtype, bias.dtype))
    y = torch.empty_like(m)   # (contiguous: m is a matrix of whole rows)
    mean, rstd = x.new_empty((2, rows), dtype=_F32).unbind()
    c, q, scale = None, None, None
    if checkpoint:
        c = _empty_checkpoint(x, rows, cols)
        q, scale = c.q.data_ptr(), c.scale.data_ptr()
    _launch(_norm_forward, device, m.data_ptr(), stride, _ptr(weight), _ptr(bias), rows, cols, code, wcode, eps, y.data_ptr(), mean.data_ptr(),
            rstd.data_ptr(), q, scale)
    return y, NormSaved(None if checkpoint else m, c, weight, bias, mean, rstd)


def layer_norm_backward(dy, saved, need_x=True, need_weight=True, need_bias=True):
    """``(dx, dweight, dbias)`` of a layer norm for the gradient ``dy`` of its output; None where not needed or where the
    norm has no weight or bias."""
    c = saved.checkpoint
    source, dtype = (saved.x, saved.x.dtype) if c is None else (c.q, c.dtype)
    device = _device(dy, "dy", source.device)
    if dy.dtype != dtype:
        raise TypeError("dy must be %s like the norm's input, not %s" % (dtype, dy.dtype))
    code = wcode = _TYPES[dtype]
    m, rows, cols, stride = _rows(dy, "dy")
    if cols != source.shape[-1] or rows != saved.mean.shape[0]:
        raise ValueError("dy must have the shape of the norm's input")
    weight, bias = saved.weight, saved.bias
    if weight is not None or bias is not None:
        wcode = _TYPES[(bias if weight is None else weight).dtype]
    dx = torch.empty_like(m) if need_x else None
    dweight = torch.empty_like(weight) if need_weight and weight is not None else None
    dbias = torch.empty_like(bias) if need_bias and bias is not None else None
    space, nbytes = None, 0
    if dweight is not None or dbias is not None:
        n = _int64()
        _check(_norm_space(rows, cols, ctypes.addressof(n)))
        nbytes = n.value
        space = dy.new_empty(nbytes, dtype=torch.uint8)
    x, x_stride, q, scale = None, 0, None, None
    if c is None:
        x, x_stride = source.data_ptr(), _rows(source, "x")[3]
    else:
        q, scale = source.data_ptr(), c.scale.data_ptr()
    _launch(_norm_backward, device, m.data_ptr(), stride, x, x_stride, q, scale, saved.mean.data_ptr(), saved.rstd.data_ptr(), _ptr(weight), rows, cols,
            code, wcode, _ptr(dx), _ptr(dweight), _ptr(dbias), _ptr(space), nbytes)
    return dx, dweight, dbias


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, checkpoint):
        y, s = layer_norm_forward(x, weight, bias, eps, checkpoint)
        c = s.checkpoint
        ctx.save_for_backward(*([s.x] if c is None else [c.q, c.scale]), s.weight, s.bias, s.mean, s.rstd)
        ctx.held, ctx.dtype = c is not None, x.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        t = list(ctx.saved_tensors)
        weight, bias, mean, rstd = t[-4:]
        c = Checkpoint8(t[0], t[1], ctx.dtype) if ctx.held else None
        saved = NormSaved(None if ctx.held else t[0], c, weight, bias, mean, rstd)
        dx, dw, db = layer_norm_backward(dy, saved, *ctx.needs_input_grad[:3])
        return dx, dw, db, None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5, checkpoint=False):
    """Layer norm over the last dimension, differentiable in ``x``, ``weight`` and ``bias``.  With ``checkpoint`` its input is
    held in 8 bits between the passes (a quarter to a half of the memory).  The gradients then are an approximation: the held values
    stand in place of the input, half a step of the checkpoint off at most, but mean and deviation remain those of the input itself
    (so a row of ``x``'s gradient adds up to zero only to that precision)."""
    return _LayerNorm.apply(x, weight, bias, eps, checkpoint)


# ---- softmax cross entropy with its projection ---------------------------------------------------------------------

def _head(x, weight, target):
    device = _device(x, "x")
    code = _type("x", x)
    _device(weight, "weight", device)
    if weight.dtype != x.dtype:
        raise TypeError("weight must be %s like x, not %s" % (x.dtype, weight.dtype))
    if not x.dim():
        raise ValueError("x has no columns")
    if weight.dim() != 2 or weight.shape[1] != x.shape[-1]:
        raise ValueError("weight must be [words, %d] for features of that width" % x.shape[-1])
    _device(target, "target", device)
    wide = target.dtype == torch.int64
    if not wide and target.dtype != torch.int32:
        raise TypeError("target must be int32 or int64, not %s" % target.dtype)
    if target.shape != x.shape[:-1]:
        raise ValueError("target must hold one word per row of x")
    m, rows, cols, stride = _rows(x, "x")
    w, vocab, _, w_stride = _rows(weight, "weight")
    t = target if target.is_contiguous() else target.contiguous()
    # (m, w and t are held here until the call: they may be copies)
    return device, (m, w, t), (m.data_ptr(), stride, w.data_ptr(), w_stride, t.data_ptr(), wide), (rows, vocab, cols, code)


def _with_space(call, device, x, args):
    """The call with a work space of the size that it asks for."""
    n = _int64()
    at = ctypes.addressof(n)
    _check(call(*args, None, at, None))
    space = x.new_empty(n.value or 1, dtype=torch.uint8)
    _launch(call, device, *args, space.data_ptr(), at)


def linear_cross_entropy_forward(x, weight, target):
    """``(loss, lse)`` per row of ``x``: minus log likelihood of the row's target word under softmax(x weight^T), and the
    logarithm of the softmax' normaliser; float32, in the shape of ``target``.  The logits are not held.  A negative target
    leaves its row out (loss 0); one beyond the vocabulary gives NaN."""
    device, held, inputs, sizes = _head(x, weight, target)
    # (two tensors of their own, not views of one: a program may change its loss in place)
    loss, lse = x.new_empty(target.shape, dtype=_F32), x.new_empty(target.shape, dtype=_F32)
    _with_space(_xent_forward, device, x, inputs + sizes + (loss.data_ptr(), lse.data_ptr()))
    return loss, lse


def linear_cross_entropy_backward(dloss, x, weight, target, lse, need_x=True, need_weight=True):
    """``(dx, dweight)`` for the gradient ``dloss`` (float32) of every row's loss; None where not needed.  ``lse`` is what the
    forward pass gave."""
    device, held, inputs, sizes = _head(x, weight, target)
    for name, v in (("dloss", dloss), ("lse", lse)):
        _device(v, name, device)
        if v.dtype != _F32 or v.shape != target.shape:
            raise ValueError("%s must be float32, one value per row of x" % name)
    dloss, lse = dloss.contiguous(), lse.contiguous()
    dx = torch.empty_like(held[0]) if need_x else None
    dweight = torch.empty_like(held[1]) if need_weight else None
    _with_space(_xent_backward, device, x, (dloss.data_ptr(),) + inputs + (lse.data_ptr(),) + sizes + (_ptr(dx), _ptr(dweight)))
    return dx, dweight


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, target):
        loss, lse = linear_cross_entropy_forward(x, weight, target)
        ctx.save_for_backward(x, weight, target, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        x, weight, target, lse = ctx.saved_tensors
        dx, dw = linear_cross_entropy_backward(dloss, x, weight, target, lse, *ctx.needs_input_grad[:2])
        return dx, dw, None


def linear_cross_entropy(x, weight, target, reduction="mean"):
    """Softmax cross entropy of ``x weight^T`` against ``target``, differentiable in ``x`` and ``weight``.  The logits are not in
    memory in either pass; their gradient is, for one piece of the vocabulary at a time (256 MB at most).  In 16-bit types that
    gradient is rounded to the type of ``x`` before the two products that follow.  Rows with a negative target are left out;
    ``reduction``: "mean" over the rows counted (0 if there is none), "sum" or "none"."""
    if reduction not in ("mean", "sum", "none"):
        raise ValueError("reduction must be mean, sum or none, not %r" % (reduction,))
    loss = _LinearCrossEntropy.apply(x, weight, target)
    if reduction == "none":
        return loss
    loss = loss.sum()
    return loss / (target >= 0).sum().clamp_(min=1) if reduction == "mean" else loss


# ---- root-mean-square norm of a residual stream -------------------------------------------------------------------------

class RmsSaved:
    """What the backward pass of a root-mean-square norm needs: the rows it is of (``x``: the sum with the residual, where there
    was one, which the stream goes on with), its weight, 1 / root mean square of every row, and the features' type."""

    __slots__ = ("x", "weight", "rstd", "dtype", "residual")

    def __init__(self, x, weight, rstd, dtype, residual):
        self.x, self.weight, self.rstd, self.dtype, self.residual = x, weight, rstd, dtype, residual


def _rms(x, weight, residual, eps, held):
    device = _device(x, "x")
    code = rcode = wcode = _type("x", x)
    m, rows, cols, stride = _rows(x, "x")
    if weight is not None:
        weight = _vector(weight, "weight", cols, device, "x")
        wcode = _type("weight", weight)
    r, r_stride, total = None, 0, None
    if residual is not None:
        _device(residual, "residual", device)
        if residual.dtype not in (x.dtype, _F32):
            raise TypeError("residual must be %s like x, or float32, not %s" % (x.dtype, residual.dtype))
        if residual.shape != x.shape:
            raise ValueError("residual must have the shape of x")
        rcode = _TYPES[residual.dtype]
        r, _, _, r_stride = _rows(residual, "residual")
        total = torch.empty_like(r)
    y, rstd, c, q, q_stride, scale = None, None, None, None, 0, None
    if held:
        c = _empty_rows8(x, rows, cols)
        q, q_stride, scale = c.q.data_ptr(), c._stride, c.scale.data_ptr()
    else:
        y = torch.empty_like(m)
        rstd = x.new_empty(rows, dtype=_F32)
    _launch(_rms_forward, device, m.data_ptr(), stride, _ptr(r), r_stride, _ptr(weight), rows, cols, code, rcode, wcode, eps, _ptr(total), _ptr(y), _ptr(rstd),
            q, q_stride, scale)
    return y, c, m if total is None else total, weight, rstd


def rms_norm_forward(x, weight=None, residual=None, eps=1e-6):
    """Root-mean-square norm of ``x + residual`` over the last dimension: ``(y, saved)``; ``saved.x`` is the sum, in the type of
    ``residual`` (that of ``x``, or float32), which the stream goes on with.  The norm is of the sum as it is held.  ``weight``: a
    vector of a floating type, its own or that of ``x``."""
    y, _, total, weight, rstd = _rms(x, weight, residual, eps, False)
    return y, RmsSaved(total, weight, rstd, x.dtype, residual is not None)


def rms_norm_backward(dy, saved, dsum=None, need_x=True, need_residual=True, need_weight=True):
    """``(dx, dresidual, dweight)`` of a root-mean-square norm for the gradient ``dy`` of its output and, where the stream goes on,
    ``dsum`` of the sum; None where not needed or not there.  Both of the first two are the gradient of the sum, in the type
    of ``x`` and of the residual: one tensor if these are the same."""
    s, rstd, weight = saved.x, saved.rstd, saved.weight
    device = _device(dy, "dy", s.device)
    if dy.dtype != saved.dtype:
        raise TypeError("dy must be %s like the norm's input, not %s" % (saved.dtype, dy.dtype))
    m, rows, cols, stride = _rows(dy, "dy")
    if dy.shape != s.shape:
        raise ValueError("dy must have the shape of the norm's input")
    d, d_stride = None, 0
    if dsum is not None:
        _device(dsum, "dsum", device)
        if dsum.dtype != s.dtype:
            raise TypeError("dsum must be %s like the sum, not %s" % (s.dtype, dsum.dtype))
        if dsum.shape != s.shape:
            raise ValueError("dsum must have the shape of the sum")
        d, _, _, d_stride = _rows(dsum, "dsum")
    need_residual = need_residual and saved.residual
    same = s.dtype == saved.dtype
    dx = torch.empty_like(m) if need_x or (same and need_residual) else None
    dresidual = torch.empty_like(m, dtype=s.dtype) if need_residual and not same else None
    dweight = torch.empty_like(weight) if need_weight and weight is not None else None
    space, nbytes = None, 0
    if dweight is not None:
        n = _int64()
        _check(_rms_space(rows, cols, ctypes.addressof(n)))
        nbytes = n.value
        space = dy.new_empty(nbytes, dtype=torch.uint8)
    code = _TYPES[saved.dtype]
    x, _, _, x_stride = _rows(s, "s")
    _launch(_rms_backward, device, m.data_ptr(), stride, _ptr(d), d_stride, x.data_ptr(), x_stride, rstd.data_ptr(), _ptr(weight), rows, cols, code,
            _TYPES[s.dtype], code if weight is None else _TYPES[weight.dtype], _ptr(dx), _ptr(dresidual), _ptr(dweight), _ptr(space), nbytes)
    return dx if need_x else None, (dx if same else dresidual) if need_residual else None, dweight


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, s = rms_norm_forward(x, weight, residual, eps)
        ctx.save_for_backward(s.x, s.weight, s.rstd)
        ctx.dtype, ctx.residual = s.dtype, s.residual
        ctx.set_materialize_grads(False)
        return (y, s.x) if s.residual else y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dsum=None):
        x, weight, rstd = ctx.saved_tensors
        need_x, need_weight, need_residual = ctx.needs_input_grad[:3]
        if dy is None:   # (only the sum was used)
            if dsum is None:
                return None, None, None, None
            return dsum.to(ctx.dtype) if need_x else None, None, dsum if need_residual else None, None
        dx, dresidual, dweight = rms_norm_backward(dy, RmsSaved(x, weight, rstd, ctx.dtype, ctx.residual), dsum, need_x, need_residual, need_weight)
        return dx, dweight, dresidual, None


def rms_norm(x, weight=None, residual=None, eps=1e-6):
    """Root-mean-square norm over the last dimension, differentiable in ``x``, ``weight`` and ``residual``: ``y``, or with a residual
    stream ``(y, sum)``, the norm of ``x + residual`` and that sum, which the stream goes on with."""
    return _RmsNorm.apply(x, weight, residual, eps)


# ---- rows in 8 bits, and logits from them -------------------------------------------------------------------------------

class Rows8:
    """A matrix in 8 bits: ``q`` (int8; rows start at multiples of 16 or 128 bytes) times ``scale`` (float32, one step
    per row, a 127th of its largest magnitude).  What ``rows8`` makes of features and weights and ``linear8`` multiplies."""

    __slots__ = ("q", "scale", "dtype", "_stride")

    def __init__(self, q, scale, dtype, stride):
        self.q, self.scale, self.dtype, self._stride = q, scale, dtype, stride

    @property
    def shape(self):
        return self.q.shape

    @staticmethod
    def of(q, scale, dtype=torch.float32):
        """Rows that were rounded elsewhere: ``q`` int8 [..., columns], ``scale`` float32 [...].  They are laid out anew, once."""
        device = _device(q, "q")
        _device(scale, "scale", device)
        if q.dtype != torch.int8 or scale.dtype != _F32:
            raise TypeError("q must be int8 and scale float32, not %s and %s" % (q.dtype, scale.dtype))
        if not q.dim() or not q.shape[-1]:
            raise ValueError("q has no columns")
        if scale.shape != q.shape[:-1]:
            raise ValueError("scale must hold one step per row of q")
        if dtype not in _TYPES:
            raise TypeError("dtype must be float32, float16 or bfloat16, not %s" % dtype)
        cols = q.shape[-1]
        wide = q.new_zeros(q.shape[:-1] + (_stride8(cols),))
        wide[..., :cols] = q
        return Rows8(wide[..., :cols], scale.contiguous(), dtype, wide.shape[-1])

    def restore(self, dtype=None):
        """The matrix, in the type it had or another floating type."""
        q = self.q
        cols = q.shape[-1]
        x = torch.empty(q.shape, dtype=dtype or self.dtype, device=q.device)
        _launch(_rows8_restore, q.device, q.data_ptr(), self._stride, self.scale.data_ptr(), q.numel() // cols, cols, _type("dtype", x), x.data_ptr())
        return x


def _stride8(cols):
    """Bytes from row to row: multiples of 128, as the caches' lines, where that adds an eighth at most, else of 16 (8192 rows of 1000
    and 141,000 words: 2.23 ms with rows of 1024 bytes, 2.50 ms with 1008, whose pieces of 128 lie on two lines each)."""
    whole = (cols + 127) // 128 * 128
    return whole if whole * 8 <= cols * 9 else (cols + 15) // 16 * 16


def _empty_rows8(x, rows, cols):
    if not cols:
        raise ValueError("x has no columns")
    stride = _stride8(cols)
    q = x.new_empty(x.shape[:-1] + (stride,), dtype=torch.int8)
    return Rows8(q if stride == cols else q[..., :cols], x.new_empty(x.shape[:-1], dtype=_F32), x.dtype, stride)


def rows8(x) -> Rows8:
    """``x`` (any shape, rows run along its last dimension) in 8 bits, one step per row: its values, no gradient goes back to it."""
    device = _device(x, "x")
    code = _type("x", x)
    m, rows, cols, stride = _rows(x, "x")
    c = _empty_rows8(x, rows, cols)
    _launch(_rows8_save, device, m.data_ptr(), stride, rows, cols, code, c.q.data_ptr(), c._stride, c.scale.data_ptr())
    return c


def _no_gradient(call, *tensors):
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError("%s has no gradient: call it under torch.no_grad(), or on detached tensors" % call)
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise ValueError("%s has no derivative in forward mode either: call it on detached tensors" % call)


def rms_norm8(x, weight=None, residual=None, eps=1e-6):
    """The output of ``rms_norm`` in 8 bits, for ``linear8``: ``(rows, sum)``; without a residual the sum is ``x``.  For serving:
    without gradients."""
    _no_gradient("rms_norm8", x, weight, residual)
    _, c, total, _, _ = _rms(x, weight, residual, eps, True)
    return c, x if residual is None else total


def linear8(x, weight, dtype=None):
    """Logits ``x weight^T`` of rows in 8 bits, ``[..., words]``.  ``x``: a ``Rows8``, or features, which are rounded by ``rows8`` first;
    ``weight``: the ``Rows8`` of a projection [words, columns].  ``dtype``: of the logits, that of ``x`` if not given.  The sums are
    exact integers.  For serving: without gradients."""
    if not isinstance(weight, Rows8):
        raise TypeError("weight must be Rows8 (rows8 of the projection), not %s" % type(weight).__name__)
    if not isinstance(x, Rows8):
        if isinstance(x, torch.Tensor):
            _no_gradient("linear8", x)
        x = rows8(x)
    xq, wq = x.q, weight.q
    device = wq.device
    if xq.device != device:
        raise ValueError("x is on %s, not on %s" % (xq.device, device))
    cols = xq.shape[-1]
    if wq.dim() != 2 or wq.shape[1] != cols:
        raise ValueError("weight must be [words, %d] for features of that width" % cols)
    words = wq.shape[0]
    out = torch.empty(xq.shape[:-1] + (words,), dtype=dtype or x.dtype, device=device)
    _launch(_linear8, device, xq.data_ptr(), x._stride, x.scale.data_ptr(), wq.data_ptr(), weight._stride, weight.scale.data_ptr(), xq.numel() // cols, words,
            cols, _type("dtype", out), out.data_ptr())
    return out


# ---- words drawn from logits ---------------------------------------------------------------------------------------------

def _limit(name, value, lead, device, types):
    """(tensor with a value per row, or None; number for all rows) of a limit."""
    if not isinstance(value, torch.Tensor):
        # (a whole number of any size: what ctypes does not hold it would wrap)
        return None, float(value) if types[0] is _F32 else max(-1, min(operator.index(value), 1 << 62))
    _device(value, name, device)
    if value.dtype not in types:
        raise TypeError("%s must be %s, not %s" % (name, " or ".join(str(t)[6:] for t in types), value.dtype))
    if value.shape != lead:
        raise ValueError("%s must be a number or hold one value per row of logits" % name)
    return (value if value.is_contiguous() else value.contiguous()), 0


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Draws a word for every row of ``logits`` [..., words] by the row's random number ``u`` (float32, within [0, 1)): ``(word, p)``,
    int64 and float32 in the shape of ``u``.  With z = (logits - their largest) / temperature, the words in falling order and equal ones
    by their number, these are left: the first ``top_k`` (0: all), of them the fewest that hold ``top_p`` of their mass, of them those of
    exp(z) >= ``min_p``.  The word is the first one, by number, at which the mass of the words left exceeds ``u`` of all of it; ``p`` is its
    share of that mass.  Temperature 0 takes the first of the largest.  Every limit is a number, or a tensor with one value per row.
    Words of logit -inf take no part; a row of which nothing is left gives -1 and 0, one with a NaN -1 and NaN.  Without gradients:
    ``p`` has none, so logits and temperatures that ask for one are refused."""
    device = _device(logits, "logits")
    _no_gradient("sample", logits, temperature if isinstance(temperature, torch.Tensor) else None)
    code = _type("logits", logits)
    m, rows, words, stride = _rows(logits, "logits")
    if not words:
        raise ValueError("logits has no words")
    lead = logits.shape[:-1]
    _device(u, "u", device)
    if u.dtype != _F32:
        raise TypeError("u must be float32, not %s" % u.dtype)
    if u.shape != lead:
        raise ValueError("u must hold one number per row of logits")
    u = u if u.is_contiguous() else u.contiguous()
    floats = (_F32,)
    temperatures, temperature = _limit("temperature", temperature, lead, device, floats)
    top_ks, top_k = _limit("top_k", top_k, lead, device, (torch.int32, torch.int64))
    top_ps, top_p = _limit("top_p", top_p, lead, device, floats)
    min_ps, min_p = _limit("min_p", min_p, lead, device, floats)
    word, p = u.new_empty(lead, dtype=torch.int64), torch.empty_like(u)
    _launch(_sample, device, m.data_ptr(), stride, rows, words, code, u.data_ptr(), _ptr(temperatures), temperature, _ptr(top_ks),
            top_ks is not None and top_ks.dtype == torch.int64, top_k, _ptr(top_ps), top_p, _ptr(min_ps), min_p, word.data_ptr(), p.data_ptr())
    return word, p
