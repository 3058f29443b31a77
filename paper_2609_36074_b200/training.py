"""Training an encoder on the cluster labels: layer norm and its gradient, cross entropy against the labels, gradient
clipping.  Argument marshalling only, like binding.py; the functions have the C entry points' names and return torch
tensors.  None of them synchronizes.

They take no part in autograd: what they return has no graph, whatever their inputs require, and the backward pass of a
model that uses them is written with layer_norm_backward and the dlogits of label_cross_entropy.  A tensor that the caller
gives to be written to (out, dlogits, the gradients that are clipped) counts as changed in place, so that autograd refuses a
backward pass for which it had saved it.

`stream`: the torch stream to work on; None is the current one.  With a stream of its own, a call allocates there and
tells the allocator that the inputs are in use there; ordering it after the work that wrote the inputs (and the outputs'
readers after it) stays with the caller, as for any torch operation."""
from __future__ import annotations

import ctypes as C
from array import array
from functools import lru_cache

from .binding import OK, lib

F32, F16, BF16 = 0, 1, 2
_INF = float("inf")


class Tensor(C.Structure):
    """Mirror of gem_nlr_tensor."""
    _fields_ = [("in_dev", C.c_void_p), ("out_dev", C.c_void_p), ("numel", C.c_int64), ("type", C.c_int32),
                ("out_type", C.c_int32)]


_fn = None          # the entry points, by name
_types = None       # torch dtype -> GEM_NLR_F32, ...
_torch = None
_written = None     # tells autograd that tensors were written to (0.3 us, 3 us for a list of 61)
_device = None      # the current device's number, and the current stream of a device as a pointer: torch's own
_stream = None      # accessors without the objects that torch.cuda.current_stream() builds (2 us of a 15 us call)


def _load():
    """The entry points with their argument types, and torch, on the first call."""
    global _fn, _types, _torch, _written, _device, _stream
    import torch
    from torch.autograd.graph import increment_version
    L = lib()
    vp, i32, i64, f32, size = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
    sig = {
        "layer_norm": [vp, i32, i64, vp, vp, i32, i64, i32, f32, vp, i64, vp, vp, vp],
        "layer_norm_backward": [vp, i64, vp, i64, i32, vp, vp, vp, i32, i64, i32, vp, i64, vp, vp, vp, size, vp],
        "layer_norm_backward_scratch_bytes": [i64, i32],
        "label_cross_entropy": [vp, i32, i64, vp, i64, i32, i32, vp, vp, vp, i64, vp, size, vp],
        "label_cross_entropy_scratch_bytes": [i64, i32],
        "clip_grad_norm": [vp, i32, f32, f32, vp, vp, size, vp],
        "clip_grad_norm_scratch_bytes": [i32],
    }
    fn = {}
    for name, args in sig.items():
        f = getattr(L, "gem_nlr_" + name)
        f.argtypes = args
        f.restype = size if name.endswith("_bytes") else C.c_int
        fn[name] = f
    _device, _stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    _written = increment_version
    _torch, _types, _fn = torch, {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}, fn
    return fn


@lru_cache(maxsize=1024)
def _scratch(name, *sizes):
    """Bytes of scratch for a call of these sizes."""
    return _fn[name](*sizes)


def _check(rc, name):
    if rc != OK:
        raise RuntimeError(f"gem_nlr_{name} failed: {rc}")


def _type(t, name):
    k = _types.get(t.dtype)
    if k is None:
        raise ValueError(f"{name} is {t.dtype}: float32, float16 or bfloat16 is needed")
    return k


def _rows(t, name):
    """(rows, columns, elements from one row to the next) of a matrix, or of a batch of them that is one."""
    if not t.is_cuda:
        raise ValueError(f"{name} is not on a GPU")
    shape = t.shape
    if len(shape) != 2:
        if not shape:
            raise ValueError(f"{name} has no columns")
        try:
            t = t.view(-1, shape[-1]) if t.numel() else t.reshape(shape[:-1].numel(), shape[-1])
        except RuntimeError:
            raise ValueError(f"the rows of {name} are not evenly spaced: make it contiguous") from None
        shape = t.shape
    n, d = shape
    ld, one = t.stride()
    if not 0 < d <= 1 << 30:
        raise ValueError(f"{name} has {d} columns")
    if one != 1 and d > 1 and n > 0:
        raise ValueError(f"the columns of {name} are not contiguous")
    return n, d, ld if n > 1 or ld > d else d


def _floats(like, n):
    """float32 of like's leading dimensions, n elements.  (empty_strided is torch's shortest way to one: 1.5 us, empty() 2.4.)"""
    if like.dim() == 2:
        return _torch.empty_strided((n,), (1,), dtype=_torch.float32, device=like.device)
    return like.new_empty(like.shape[:-1], dtype=_torch.float32)


def _vector(t, d, at, name):
    if t.shape != (d,) or not t.is_contiguous() or t.get_device() != at:
        raise ValueError(f"{name} has to be a contiguous vector of {d} on GPU {at}")
    return t.data_ptr()


def _there(fn, stream, inputs, *args):
    """The call on another stream than the current one, or on a device that is not current."""
    torch = _torch
    device = inputs[0].device
    if stream is None:
        with torch.cuda.device(device):
            return fn(*args)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the data on {device}")
    with torch.cuda.stream(stream):
        got = fn(*args)
    for t in inputs:
        if t is not None and t.is_cuda:
            t.record_stream(stream)
    return got


def _given(out, like, name):
    """The row distance of an output that the caller gave."""
    if out.shape != like.shape or out.dtype != like.dtype or out.device != like.device:
        raise ValueError(f"{name} has to be {tuple(like.shape)} {like.dtype} on {like.device}")
    return _rows(out, name)[2]


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """gem_nlr_layer_norm over the last dimension: (y, mean, rstd), y of x's type and shape, mean and rstd float32 of
    x's leading dimensions.  weight, bias: float32 or x's type, None for ones and zeros."""
    fn = _fn or _load()
    n, d, ld = _rows(x, "x")
    at = x.get_device()
    if stream is not None or at != _device():
        return _there(layer_norm, stream, (x, weight, bias, out), x, weight, bias, eps, out)
    torch = _torch
    t = wt = _type(x, "x")
    wp = bp = None
    if weight is not None:
        wt, wp = _type(weight, "weight"), _vector(weight, d, at, "weight")
    if bias is not None:
        bt, bp = _type(bias, "bias"), _vector(bias, d, at, "bias")
        if weight is None:
            wt = bt
        elif bt != wt:
            raise ValueError(f"weight is {weight.dtype} and bias {bias.dtype}")
    if wt != t and wt != F32:
        raise ValueError("weight and bias have to be float32 or of x's type")
    if not 0 <= eps < _INF:
        raise ValueError(f"eps is {eps}")
    if out is None:
        y, ldy = torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape), d
    else:
        y, ldy = out, _given(out, x, "out")
    mean = _floats(x, n)
    rstd = torch.empty_like(mean)
    _check(fn["layer_norm"](x.data_ptr(), t, ld, wp, bp, wt, n, d, eps, y.data_ptr(), ldy, mean.data_ptr(), rstd.data_ptr(),
                            _stream(at)), "layer_norm")
    if out is not None:
        _written(out)
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, need_dx=True, need_dweight=None, need_dbias=None, stream=None):
    """gem_nlr_layer_norm_backward: (dx, dweight, dbias), None for each that is not needed.  dx has x's type and shape,
    dweight and dbias the weight's type (float32 without a weight).  By default the gradients of weight and bias are
    taken where there is a weight."""
    fn = _fn or _load()
    n, d, ld = _rows(x, "x")
    at = x.get_device()
    if stream is not None or at != _device():
        return _there(layer_norm_backward, stream, (x, dy, mean, rstd, weight), dy, x, mean, rstd, weight, need_dx, need_dweight,
                      need_dbias)
    torch = _torch
    if dy.shape != x.shape or dy.dtype != x.dtype or dy.get_device() != at:
        raise ValueError(f"dy has to be {tuple(x.shape)} {x.dtype} on GPU {at}, as x")
    ldg = _rows(dy, "dy")[2]
    for s, name in ((mean, "mean"), (rstd, "rstd")):
        if s.dtype != torch.float32 or s.numel() != n or not s.is_contiguous() or s.get_device() != at:
            raise ValueError(f"{name} has to be {n} contiguous float32 on GPU {at}")
    t = _type(x, "x")
    wt, wp = F32, None
    if weight is not None:
        wt, wp = _type(weight, "weight"), _vector(weight, d, at, "weight")
        if wt != t and wt != F32:
            raise ValueError("weight has to be float32 or of x's type")
    if need_dweight is None:
        need_dweight = weight is not None
    if need_dbias is None:
        need_dbias = weight is not None
    if not (need_dx or need_dweight or need_dbias):
        return None, None, None
    dx = dw = db = None
    if need_dx:
        dx = torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)
    if need_dweight:
        dw = mean.new_empty(d) if weight is None else torch.empty_like(weight)
    if need_dbias:
        db = mean.new_empty(d) if weight is None else torch.empty_like(weight)
    size = _scratch("layer_norm_backward_scratch_bytes", n, d)
    scratch = mean.new_empty(size, dtype=torch.uint8) if size else mean
    _check(fn["layer_norm_backward"](
        dy.data_ptr(), ldg, x.data_ptr(), ld, t, mean.data_ptr(), rstd.data_ptr(), wp, wt, n, d,
        None if dx is None else dx.data_ptr(), d, None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
        scratch.data_ptr(), size, _stream(at)), "layer_norm_backward")
    return dx, dw, db


def label_cross_entropy(logits, labels, mean=True, dlogits=None, need_grad=True, stream=None):
    """gem_nlr_label_cross_entropy: (loss, row_loss, dlogits).  logits: (n, k); labels: n int32 as GemNlr.labels gives
    them, negative ones left out.  loss: a float32 scalar, the mean over the rows that count (mean=False: the sum);
    row_loss: n float32; dlogits: the loss's gradient in logits' type, written to the tensor given (the logits themselves
    are fine) or a new one; need_grad=False: None."""
    fn = _fn or _load()
    n, k, ld = _rows(logits, "logits")
    at = logits.get_device()
    if stream is not None or at != _device():
        return _there(label_cross_entropy, stream, (logits, labels, dlogits), logits, labels, mean, dlogits, need_grad)
    torch = _torch
    t = _type(logits, "logits")
    lead = logits.shape[:-1]
    if labels.dtype != torch.int32 or labels.shape != lead or not labels.is_contiguous() or labels.get_device() != at:
        raise ValueError(f"labels have to be {tuple(lead)} contiguous int32 on GPU {at}")
    ldd, dp, given = k, None, None
    if not need_grad:
        dlogits = None
    else:
        if dlogits is None:
            dlogits = torch.empty_like(logits) if logits.is_contiguous() else logits.new_empty(logits.shape)
        else:
            given, ldd = dlogits, _given(dlogits, logits, "dlogits")
        dp = dlogits.data_ptr()
    row = _floats(logits, n)
    loss = torch.empty_strided((), (), dtype=torch.float32, device=logits.device)
    size = _scratch("label_cross_entropy_scratch_bytes", n, k)
    scratch = labels.new_empty(size, dtype=torch.uint8) if size else labels          # (none is needed then)
    _check(fn["label_cross_entropy"](logits.data_ptr(), t, ld, labels.data_ptr(), n, k, 1 if mean else 0, loss.data_ptr(), row.data_ptr(),
                                     dp, ldd, scratch.data_ptr(), size, _stream(at)), "label_cross_entropy")
    if given is not None:
        _written(given)
    return loss, row, dlogits


def _norm_and_clip(grads, max_norm, out, eps, stream):
    fn = _fn or _load()
    torch = _torch
    if not grads:
        raise ValueError("no tensors")
    if not grads[0].is_cuda:
        raise ValueError("the first tensor is not on a GPU")
    at = grads[0].get_device()
    if stream is not None or at != _device():
        return _there(_norm_and_clip, stream, grads if out is None or out is grads else grads + out, grads, max_norm, out, eps, None)
    count, types = len(grads), _types
    if out is not None:
        if len(out) != count:
            raise ValueError(f"{count} tensors and {len(out)} outputs")
        if not max_norm >= 0:
            raise ValueError(f"max_norm is {max_norm}")
        if not eps >= 0:
            raise ValueError(f"eps is {eps}")
    kinds, sizes, ptrs = [types.get(g.dtype) for g in grads], [g.numel() for g in grads], [g.data_ptr() for g in grads]
    if None in kinds or [g.get_device() for g in grads].count(at) != count:
        raise ValueError(f"every tensor has to be float32, float16 or bfloat16 on GPU {at}")
    whole = [g.is_contiguous() for g in grads]
    for i in (i for i, w in enumerate(whole) if not w):
        if not _dense(grads[i]):
            raise ValueError(f"tensor {i} has gaps between its elements")
    to, to_kinds = ptrs, kinds
    if out is None:
        to = [0] * count
    elif out is not grads:
        to, to_kinds = [o.data_ptr() for o in out], [types.get(o.dtype) for o in out]
        if [o.numel() for o in out] != sizes or [o.get_device() for o in out].count(at) != count or \
                (to_kinds != kinds and any(o != k and o != F32 for o, k in zip(to_kinds, kinds))):
            raise ValueError(f"every output has to have its tensor's size and type, or float32, on GPU {at}")
        if False in whole or False in [o.is_contiguous() for o in out]:
            for i, (g, o) in enumerate(zip(grads, out)):
                if not (g.is_contiguous() and o.is_contiguous()) and (o.shape != g.shape or o.stride() != g.stride() or not _dense(o)):
                    raise ValueError(f"the elements of output {i} are in another order than its tensor's")
    flat = [0] * (4 * count)                         # gem_nlr_tensor as four 64-bit words
    flat[0::4], flat[1::4], flat[2::4] = ptrs, to, sizes
    flat[3::4] = [k | o << 32 for k, o in zip(kinds, to_kinds)]
    table = array("Q", flat)
    norm = torch.empty_strided((), (), dtype=torch.float32, device=grads[0].device)
    size = _scratch("clip_grad_norm_scratch_bytes", count)
    scratch = norm.new_empty(size // 4)
    _check(fn["clip_grad_norm"](table.buffer_info()[0], count, max_norm, eps, norm.data_ptr(), scratch.data_ptr(), size, _stream(at)), "clip_grad_norm")
    if out is not None:
        _written(out)
    return norm


def _dense(t):
    """Whether the tensor's elements fill its memory, in any order of its dimensions."""
    need = 1
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size != 1:
            if stride != need:
                return False
            need *= size
    return True


def clip_grad_norm(grads, max_norm, out=None, eps=1e-6, stream=None):
    """gem_nlr_clip_grad_norm: scales all tensors by min(1, max_norm / (norm + eps)), in place or into `out` (tensors of
    the same sizes, in the same order of elements, of the same types or float32), and returns the norm before it, a float32
    scalar on the GPU."""
    grads = list(grads)
    return _norm_and_clip(grads, max_norm, grads if out is None else list(out), eps, stream)


def grad_norm(grads, stream=None):
    """The same norm alone; nothing else is written."""
    return _norm_and_clip(list(grads), 0.0, None, 0.0, stream)
