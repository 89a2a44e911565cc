"""Training-node operators on device tensors: argument checks and marshalling only.

The nodes of a transformer training graph that a rematerialization schedule
computes again first, with their gradients as calls (nodes) of their own:

  dropout, dropout_backward           counter-based, the mask never stored
  layer_norm, layer_norm_backward     with the dropout and residual sum before it
  softmax, softmax_backward           scale, masks, softmax and dropout of scores

A call made again with the same inputs gives the same bits, in whatever stage
of a plan it runs. Every computation is a HIP kernel of libckm (include/ckm.h
states each operator's definition); there is no other implementation to fall
back to. Tensors are float32, float16 or bfloat16 on the current device.

Calls enqueue kernels on `stream` (a torch.cuda.Stream; None: the current one)
and return at once. With a stream other than the current one, that stream first
waits for what the current stream holds at the call, so arguments made on the
current stream are whole when they are read, and their memory is not given out
again before the call is through with it: they may be dropped at once. Work on
any third stream is the caller's to order, as are later uses of the arguments
on other streams. Results that a call allocates belong to its stream. (To order
everything oneself, make the stream the current one and leave `stream` out.)

No call records an autograd graph, whatever its tensors require: results that it
allocates require no gradient, and gradients are the *_backward calls.
"""
from __future__ import annotations

import ctypes as C
import functools
import math

import torch

from . import ckm

F32, F16, BF16 = range(3)
SCORES_CAUSAL = 1
MASK_NONE, MASK_BOOL, MASK_ADD = range(3)
MAX_ROWS, MAX_COLS, MAX_NORM_COLS = 0x7fffffff, 1 << 30, 32768
_TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}


class _Drop(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("site", C.c_uint64), ("d_site", C.c_void_p), ("keep", C.c_uint32)]


class _Scores(C.Structure):
    _fields_ = [("batch", C.c_int64), ("heads", C.c_int64), ("queries", C.c_int64), ("keys", C.c_int64),
                ("scale", C.c_float), ("flags", C.c_uint32), ("d_lengths", C.c_void_p), ("d_mask", C.c_void_p),
                ("mask_kind", C.c_int32), ("mask_stride", C.c_int64 * 3)]


_Stride = C.c_int64 * 3


class Dropout:
    """Which elements a dropout keeps, as a function of (seed, site, row, column) alone.

    p: drop probability, kept to 16 bits (an element is kept with probability
    keep / 65536, keep = floor((1 - p) 65536), and scaled by its inverse).
    site: names the place and step; equal (seed, site) give equal masks.
    d_site: an int64 device tensor of one element, added to site when a kernel
    runs: the step counter of a captured graph.
    p, seed, site and d_site can be assigned; later calls go by the new values."""

    __slots__ = ("_p", "_d_site", "_c")

    def __init__(self, p: float, seed: int, site: int = 0, d_site=None):
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in [0, 1], got %r" % (p,))
        if not 0 <= seed < 1 << 64 or not 0 <= site < 1 << 64:
            raise ValueError("seed and site must be unsigned 64-bit numbers, got %r and %r" % (seed, site))
        self._p, self._d_site = float(p), None
        self._c = _Drop(int(seed), int(site), None, math.floor((1.0 - self._p) * 65536.0))
        if d_site is not None:
            self.d_site = d_site

    def __reduce__(self):   # a copy has values of its own
        return Dropout, (self.p, self.seed, self.site, self.d_site)

    @property
    def p(self) -> float:
        return self._p

    @p.setter
    def p(self, p: float):
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in [0, 1], got %r" % (p,))
        self._p = float(p)
        self._c.keep = math.floor((1.0 - self._p) * 65536.0)

    @property
    def keep(self) -> int:
        return self._c.keep

    @property
    def seed(self) -> int:
        return self._c.seed

    @seed.setter
    def seed(self, seed: int):
        if not 0 <= seed < 1 << 64:
            raise ValueError("seed must be an unsigned 64-bit number, got %r" % (seed,))
        self._c.seed = int(seed)

    @property
    def site(self) -> int:
        return self._c.site

    @site.setter
    def site(self, site: int):
        if not 0 <= site < 1 << 64:
            raise ValueError("site must be an unsigned 64-bit number, got %r" % (site,))
        self._c.site = int(site)

    @property
    def d_site(self):
        return self._d_site

    @d_site.setter
    def d_site(self, d_site):
        if d_site is not None and (not isinstance(d_site, torch.Tensor) or not d_site.is_cuda
                                   or d_site.dtype != torch.int64 or d_site.numel() != 1):
            raise ValueError("d_site must be an int64 device tensor of one element")
        self._d_site = d_site
        self._c.d_site = None if d_site is None else d_site.data_ptr()


def _tensor(t, name: str, dtype=None, device=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if dtype is None:
        if t.dtype not in _TYPES:
            raise ValueError("%s must be float32, float16 or bfloat16, got %s" % (name, t.dtype))
    elif t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if device is None:
        if t.get_device() != torch.cuda.current_device():
            raise ValueError("%s is on %s, not on the current device" % (name, t.device))
    elif t.get_device() != device:
        raise ValueError("%s is on %s, not on device %d" % (name, t.device, device))
    return t


def _rows(t, name: str, shape, dtype, device):
    """(pointer, row stride) of a tensor of `shape` seen as rows of its last dimension; (None, 0) for None."""
    if t is None:
        return None, 0
    # the common case first: what is a tensor, and on which device, one call tells
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == shape:
        if t.is_contiguous() or t.numel() == 0:
            return t.data_ptr(), shape[-1]
    else:
        _tensor(t, name, dtype, device)
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("%s: the last dimension must be contiguous, got strides %s" % (name, t.stride()))
    # the other dimensions as one: each stride spans the next inner dimension
    ld, span = None, 1
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if ld is None:
            ld, span = s, n * s
        elif s == span:
            span = n * s
        else:
            raise ValueError("%s: rows must lie at one stride, got shape %s, strides %s (make it contiguous)"
                             % (name, tuple(t.shape), t.stride()))
    return t.data_ptr(), shape[-1] if ld is None else ld


def _vector(t, name: str, cols: int, dtype, device):
    if t is None:
        return None
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == (cols,)
            and t.is_contiguous()):
        return t.data_ptr()
    _tensor(t, name, dtype, device)
    if t.dim() != 1 or t.shape[0] != cols or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d elements, got shape %s" % (name, cols, tuple(t.shape)))
    return t.data_ptr()


def _drop_ptr(drop, device):
    if drop is None:
        return None
    if not isinstance(drop, Dropout):
        raise ValueError("drop must be an ops.Dropout, got %s" % type(drop).__name__)
    if drop._d_site is not None and drop._d_site.get_device() != device:
        raise ValueError("d_site is on %s, not on device %d" % (drop._d_site.device, device))
    return C.byref(drop._c)


# the current stream's pointer without a torch.cuda.Stream object around it (0.1 us instead of 2.8), and
# the current device's number
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on(stream, drop, *tensors):
    """The context of a call on `stream`, once that stream waits for the current one and holds the call's tensors."""
    here = torch.cuda.current_stream(stream.device)
    if stream != here:
        within = torch.cuda.is_current_stream_capturing()
        with torch.cuda.stream(stream):
            # a capture cannot wait for work that is not part of it
            if within or not torch.cuda.is_current_stream_capturing():
                stream.wait_stream(here)
        for t in (*tensors, drop.d_site if isinstance(drop, Dropout) else None):
            if isinstance(t, torch.Tensor) and t.device == stream.device:
                t.record_stream(stream)
    return torch.cuda.stream(stream)


def _like(t):
    """A contiguous tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _first(t, name: str):
    """(device, shape, type, columns, rows, pointer, row stride) of an operator's first tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in _TYPES or t.get_device() != _current_device():
        _tensor(t, name)
    shape = t.shape
    if not shape:
        raise ValueError("%s must have at least one dimension" % name)
    cols, device = shape[-1], t.get_device()
    rows = t.numel() // cols if cols else shape[:-1].numel()
    p, ld = (t.data_ptr(), cols) if t.is_contiguous() else _rows(t, name, shape, t.dtype, device)
    return device, shape, t.dtype, cols, rows, p, ld


def dropout(x, drop: Dropout, residual=None, out=None, stream=None):
    """y = residual + D(x), rows by the last dimension (ckm_dropout_async). out may be x or residual.
    Outside autograd: the gradient is dropout_backward."""
    if stream is not None:
        with _on(stream, drop, x, residual, out):
            return dropout(x, drop, residual, out)
    device, shape, dtype, cols, rows, xp, ldx = _first(x, "x")
    if drop is None:
        raise ValueError("drop is needed")
    rp, ldr = _rows(residual, "residual", shape, dtype, device)
    if out is None:
        y = _like(x)
        yp, ldy = y.data_ptr(), cols
    else:
        y = out
        yp, ldy = _rows(y, "out", shape, dtype, device)
    ckm._check(ckm.lib().ckm_dropout_async(_TYPES[dtype], rows, cols, xp, ldx, rp, ldr, _drop_ptr(drop, device), yp, ldy,
                                           _raw_stream(device)))
    return y


def dropout_backward(dy, drop: Dropout, out=None, stream=None):
    """The gradient of x: D(dy). (The residual's gradient is dy.)"""
    return dropout(dy, drop, out=out, stream=stream)


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, residual=None, drop: Dropout = None, out=None,
               stream=None):
    """(y, h, stats) of the layer norm over the last dimension (ckm_layer_norm_async).

    h = residual + D(x), rounded to x's type; x itself when neither is given.
    weight, bias: vectors of x's type or float32, both of one type. stats:
    float32 [..., 2], mean and 1 / standard deviation of each row of h.
    out: for y; may be x or residual. With y in the place of an x that would be
    h, h is None: keep x for layer_norm_backward, which is the gradient (the
    call is outside autograd)."""
    if stream is not None:
        with _on(stream, drop, x, weight, bias, residual, out):
            return layer_norm(x, weight, bias, eps, residual, drop, out)
    device, shape, dtype, cols, rows, xp, ldx = _first(x, "x")
    wt = weight.dtype if weight is not None else bias.dtype if bias is not None else dtype
    if wt is not dtype and wt is not torch.float32:
        raise ValueError("weights must be %s or float32, got %s" % (dtype, wt))
    wp, bp = _vector(weight, "weight", cols, wt, device), _vector(bias, "bias", cols, wt, device)
    rp, ldr = _rows(residual, "residual", shape, dtype, device)
    if out is None:
        y = _like(x)
        yp, ldy = y.data_ptr(), cols
    else:
        y = out
        yp, ldy = _rows(y, "out", shape, dtype, device)
    if residual is None and drop is None:
        h, hp = None if yp == xp and rows else x, None
    else:
        h = _like(x)
        hp = h.data_ptr()
    stats = x.new_empty(shape[:-1] + (2,), dtype=torch.float32)
    ckm._check(ckm.lib().ckm_layer_norm_async(_TYPES[dtype], _TYPES[wt], rows, cols, xp, ldx, rp, ldr,
                                              _drop_ptr(drop, device), wp, bp, eps, hp, cols, yp, ldy,
                                              stats.data_ptr(), _raw_stream(device)))
    return y, h, stats


def layer_norm_backward(dy, h, stats, weight=None, dres=None, drop: Dropout = None, wtype=None, out=None, work=None,
                        stream=None):
    """(dx, dh, dweight, dbias) of layer_norm (ckm_layer_norm_backward_async).

    h, stats: what layer_norm returned. dres: a gradient that reaches h past the
    norm, added to dh. drop: the forward call's; dx = D(dh), and without one dx
    is dh. dweight and dbias are of weight's type (wtype when there is none:
    x's type or float32). out: for dh; may be dy, h or dres. work: a uint8
    device buffer of layer_norm_workspace(rows, cols) bytes to use."""
    if stream is not None:
        with _on(stream, drop, dy, h, stats, weight, dres, out, work):
            return layer_norm_backward(dy, h, stats, weight, dres, drop, wtype, out, work)
    device, shape, dtype, cols, rows, dyp, lddy = _first(dy, "dy")
    wt = weight.dtype if weight is not None else wtype or dtype
    if wt is not dtype and wt is not torch.float32:
        raise ValueError("weights must be %s or float32, got %s" % (dtype, wt))
    wp = _vector(weight, "weight", cols, wt, device)
    _stats(stats, shape, device)
    hp, ldh = _rows(h, "h", shape, dtype, device)
    rp, ldr = _rows(dres, "dres", shape, dtype, device)
    if out is None:
        dh = _like(dy)
        op, ldo = dh.data_ptr(), cols
    else:
        dh = out
        op, ldo = _rows(dh, "out", shape, dtype, device)
    if drop is None:
        dx, xp = dh, None
    else:
        dx = _like(dy)
        xp = dx.data_ptr()
    if weight is not None:
        dw, db = torch.empty_like(weight), torch.empty_like(weight)
    else:
        dw, db = torch.empty((2, cols), dtype=wt, device=dy.device).unbind(0)
    wkp, wkb, work = _work(work, layer_norm_workspace(rows, cols), dy)
    ckm._check(ckm.lib().ckm_layer_norm_backward_async(
        _TYPES[dtype], _TYPES[wt], rows, cols, dyp, lddy, hp, ldh, stats.data_ptr(), wp, rp, ldr,
        _drop_ptr(drop, device), op, ldo, xp, cols, dw.data_ptr(), db.data_ptr(), wkp, wkb, _raw_stream(device)))
    return dx, dh, dw, db


@functools.lru_cache(maxsize=1024)
def layer_norm_workspace(rows: int, cols: int) -> int:
    """Bytes of work buffer that layer_norm_backward needs (ckm_layer_norm_workspace_size)."""
    out = C.c_size_t()
    ckm._check(ckm.lib().ckm_layer_norm_workspace_size(rows, cols, C.byref(out)))
    return out.value


@functools.lru_cache(maxsize=1024)
def softmax_workspace(batch: int, heads: int, queries: int, keys: int) -> int:
    """Bytes of work buffer that softmax and softmax_backward need (ckm_softmax_workspace_size)."""
    out = C.c_size_t()
    ckm._check(ckm.lib().ckm_softmax_workspace_size(C.byref(_Scores(batch, heads, queries, keys)), C.byref(out)))
    return out.value


def _stats(stats, shape, device):
    _tensor(stats, "stats", torch.float32, device)
    if stats.shape != shape[:-1] + (2,) or not stats.is_contiguous():
        raise ValueError("stats must be contiguous of shape %s, got %s" % (tuple(shape[:-1]) + (2,), tuple(stats.shape)))


def _work(work, need: int, like):
    """(pointer, bytes, tensor) of the caller's work buffer, or of one made for the call on its stream."""
    if work is None:
        if not need:
            return None, 0, None
        work = like.new_empty(need, dtype=torch.uint8)
    else:
        _tensor(work, "work", torch.uint8, like.get_device())
        if not work.is_contiguous():
            raise ValueError("work must be contiguous")
    return work.data_ptr(), work.numel(), work


def _strides(t, name: str, shape, dtype, device):
    """(pointer, strides of batch, heads, queries) of a tensor of shape `shape`, up to four dimensions."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == shape):
        _tensor(t, name, dtype, device)
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    s = t.stride()
    if shape[-1] > 1 and s[-1] != 1 and t.numel():
        raise ValueError("%s: the last dimension must be contiguous, got strides %s" % (name, s))
    return t.data_ptr(), _Stride(*((0,) * (4 - len(s)) + s[:-1]))


def _scores(scores, scale, causal, lengths, mask):
    """The C struct of a call's shape, scale and masks, with the tensors it points to."""
    if (not isinstance(scores, torch.Tensor) or not scores.is_cuda or scores.dtype not in _TYPES
            or scores.get_device() != _current_device()):
        _tensor(scores, "scores")
    device, shape = scores.get_device(), scores.shape
    if not 1 <= len(shape) <= 4:
        raise ValueError("scores must have one to four dimensions, got shape %s" % (tuple(shape),))
    c = _Scores(*(1,) * (4 - len(shape)), *shape, scale, SCORES_CAUSAL if causal else 0)
    if lengths is not None:
        _tensor(lengths, "lengths", torch.int32, device)
        if lengths.numel() != c.batch or not lengths.is_contiguous():
            raise ValueError("lengths must hold %d contiguous elements, got shape %s" % (c.batch, tuple(lengths.shape)))
        c.d_lengths = lengths.data_ptr()
    if mask is not None:
        if not isinstance(mask, torch.Tensor) or mask.dtype not in (torch.bool, torch.uint8, scores.dtype):
            raise ValueError("mask must be a bool, uint8 or %s device tensor" % scores.dtype)
        _tensor(mask, "mask", mask.dtype, device)
        try:
            mask = mask.expand(scores.shape)
        except RuntimeError:
            raise ValueError("mask of shape %s does not broadcast to scores of shape %s"
                             % (tuple(mask.shape), tuple(scores.shape))) from None
        if shape[-1] > 1 and mask.stride(-1) == 0:
            raise ValueError("mask must have each of the %d keys in its last dimension: it is broadcast over queries, "
                             "heads and batches alone" % shape[-1])
        c.d_mask, c.mask_stride = _strides(mask, "mask", scores.shape, mask.dtype, device)
        c.mask_kind = MASK_ADD if mask.dtype == scores.dtype else MASK_BOOL
    return c, device


def softmax(scores, scale: float = 1.0, causal: bool = False, lengths=None, mask=None, drop: Dropout = None, out=None,
            work=None, stream=None):
    """(probabilities, stats) of attention scores [batch, heads, queries, keys] (ckm_softmax_async).

    Fewer dimensions stand for leading ones of 1. lengths: int32 [batch], the
    keys that each sequence has. causal: query i sees key j iff j <= i + keys -
    queries. mask: bool or uint8 (0 hides a key) or of the scores' type (added
    after the scale; -inf hides), with every key in its last dimension and
    broadcast over queries, heads and batches. A row that sees nothing gives
    zeros. stats: float32 [..., queries, 2], the largest logit and 1 / the sum
    of exponentials. out: for the probabilities; may be scores (which
    softmax_backward, the gradient, needs: the call is outside autograd). work:
    a uint8 device buffer of softmax_workspace(...) bytes to use."""
    if stream is not None:
        with _on(stream, drop, scores, lengths, mask, out, work):
            return softmax(scores, scale, causal, lengths, mask, drop, out, work)
    c, device = _scores(scores, scale, causal, lengths, mask)
    shape, dtype = scores.shape, scores.dtype
    xp, xs = _strides(scores, "scores", shape, dtype, device)
    if out is None:
        y = _like(scores)
        yp, ys = y.data_ptr(), _Stride(c.heads * c.queries * c.keys, c.queries * c.keys, c.keys)
    else:
        y = out
        yp, ys = _strides(y, "out", shape, dtype, device)
    stats = scores.new_empty(shape[:-1] + (2,), dtype=torch.float32)
    wp, wb, work = _work(work, softmax_workspace(c.batch, c.heads, c.queries, c.keys), scores)
    ckm._check(ckm.lib().ckm_softmax_async(_TYPES[dtype], C.byref(c), xp, xs, _drop_ptr(drop, device), yp, ys,
                                           stats.data_ptr(), wp, wb, _raw_stream(device)))
    return y, stats


def softmax_backward(dy, scores, stats, scale: float = 1.0, causal: bool = False, lengths=None, mask=None,
                     drop: Dropout = None, out=None, work=None, stream=None):
    """The scores' gradient (ckm_softmax_backward_async): the forward call's scores, stats, masks and drop.
    out: may be dy or scores."""
    if stream is not None:
        with _on(stream, drop, dy, scores, stats, lengths, mask, out, work):
            return softmax_backward(dy, scores, stats, scale, causal, lengths, mask, drop, out, work)
    c, device = _scores(scores, scale, causal, lengths, mask)
    shape, dtype = scores.shape, scores.dtype
    _stats(stats, shape, device)
    gp, gs = _strides(dy, "dy", shape, dtype, device)
    xp, xs = _strides(scores, "scores", shape, dtype, device)
    if out is None:
        dx = _like(scores)
        op, os_ = dx.data_ptr(), _Stride(c.heads * c.queries * c.keys, c.queries * c.keys, c.keys)
    else:
        dx = out
        op, os_ = _strides(dx, "out", shape, dtype, device)
    wp, wb, work = _work(work, softmax_workspace(c.batch, c.heads, c.queries, c.keys), scores)
    ckm._check(ckm.lib().ckm_softmax_backward_async(_TYPES[dtype], C.byref(c), gp, gs, xp, xs, stats.data_ptr(),
                                                    _drop_ptr(drop, device), op, os_, wp, wb, _raw_stream(device)))
    return dx
