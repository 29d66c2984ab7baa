"""Operators on rows held in 8 bits (include/comp_ams_rows8.h): the root-mean-square norm with the residual's addition and an output in
8 bits, activation checkpoints in 8 bits, weight gradients formed from them per worker, and the product of 8-bit integers with a scale for
each token and channel.  Conventions are those of operators.py.

A row in 8 bits is q (int8) and one float32 scale: q = rint(x / scale), scale = absmax / 127, or with binary=True the least power of two
not below that, which makes q * scale exact in every type whose range holds it.

    q, scale, h, rstd = rms_norm_q8(x, gain, residual, binary=True)         # 8 bits for the product, and kept for the backward pass
    y = linear_q8(q, scale, wq, wscale)                                     # wq, wscale = quantize_rows(weight)
    linear_weight_grad(dy, q, scale, grads[:, a:b].unflatten(1, (outs, cols)), binary=True)
    dx = rms_norm_backward(dx_product, h, rstd, gain, grads[:, c:c + cols], dresidual=dh)
"""
from __future__ import annotations

from .binding import lib
from .operators import _check, _like, _need, _param_grad, _rows, _type, _work_bytes

# Small calls cost what the host does for them, so the common case (dense tensors on the current GPU) takes short ways here: torch and
# the library are looked up once, and a tensor is asked once for what it knows.
_torch = _lib = None


def _load():
    global _torch, _lib
    import torch
    _lib = lib()
    _torch = torch


def _with_stream(stream, call, *args, **kw):
    """The call with that raw stream as torch's current one, so that what it allocates belongs to it."""
    with _torch.cuda.stream(_torch.cuda.ExternalStream(stream)):
        return call(*args, **kw)


def _stream(like, *tensors):
    """The raw current stream; all tensors must be on the GPU of `like`, which has to be the current one."""
    dev = like.get_device()
    if dev < 0:
        raise ValueError("tensors must be on the GPU")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("all tensors must be on the same GPU")
    if dev != _torch._C._cuda_getDevice():
        raise ValueError(f"the tensors are on GPU {dev}, which is not the current one")
    return _torch._C._cuda_getCurrentRawStream(dev)


def _columns(t, what):
    """(columns, row stride) of a tensor [..., columns] whose rows are evenly spaced and dense."""
    if t.is_contiguous() and t.dim():
        cols = t.shape[-1]
        return cols, cols
    return _rows(t, what)[1:]


def _new(t, dtype=None):
    """A dense tensor of t's shape (empty_like takes two thirds of new_empty's time, and keeps strides)."""
    if t.is_contiguous():
        return _torch.empty_like(t) if dtype is None else _torch.empty_like(t, dtype=dtype)
    return t.new_empty(t.shape, dtype=dtype)


def _bytes(t, what):
    """_columns of an int8 tensor."""
    if t.dtype is not _torch.int8:
        raise ValueError(f"{what} must be int8")
    return _columns(t, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _scales(t, lead, what):
    """Of a dense float32 tensor with the leading dimensions `lead`: how many numbers it has, one a row."""
    if t.shape != lead or t.dtype is not _torch.float32 or not t.is_contiguous():
        raise ValueError(f"{what} must be a dense float32 tensor with one number for each row")
    return t.numel()


def _parameter(t, size, what):
    if t.dtype is not _torch.float32 or t.numel() != size or not t.is_contiguous():
        raise ValueError(f"{what} must be a dense float32 tensor of {size} elements")


def _memory(like, name, *args):
    """(work tensor or None, pointer, bytes) for the size that the library asks for."""
    need = _work_bytes(name, *args)
    if need == 0:
        return None, None, 0
    w = like.new_empty(need, dtype=_torch.uint8)
    return w, w.data_ptr(), need


def _sixteens(t, stride):
    """Whether an int8 or 16-bit array is known to have its rows at multiples of 16 bytes."""
    return 1 if (t.data_ptr() | stride * t.element_size()) % 16 == 0 and stride < 1 << 22 else 0


def quantize_rows(x, binary=False, *, stream=None):
    """x [..., cols] (float32, bfloat16 or float16) in 8 bits: (q int8 of its shape, scale float32 of its leading dimensions).  A row with a
    NaN or an infinity has the scale NaN."""
    if _torch is None:
        _load()
    if stream is not None:
        return _with_stream(stream, quantize_rows, x, binary)
    kind = _type(x)
    cols, x_stride = _columns(x, "x")
    s = _stream(x)
    q = _new(x, _torch.int8)
    scale = x.new_empty(x.shape[:-1], dtype=_torch.float32)
    rc = _lib.comp_ams_quantize_rows(q.data_ptr(), scale.data_ptr(), x.data_ptr(), scale.numel(), cols, cols, x_stride, 1 if binary else 0, kind, s)
    if rc:
        _check(rc)
    return q, scale


def restore_rows(q, scale, dtype=None, out=None, *, stream=None):
    """q * scale in `dtype` (float32 if neither it nor out is given), rounded once."""
    if _torch is None:
        _load()
    if stream is not None:
        return _with_stream(stream, restore_rows, q, scale, dtype, out)
    cols, q_stride = _bytes(q, "q")
    shape = q.shape
    rows = _scales(scale, shape[:-1], "scale")
    s = _stream(q, scale, out)
    if out is None:
        out = _new(q, _torch.float32 if dtype is None else dtype)
        stride = cols
    else:
        _need(out.shape == shape and dtype in (None, out.dtype), "out must have the shape of q and the type asked for")
        stride = _columns(out, "out")[1]
    rc = _lib.comp_ams_restore_rows(out.data_ptr(), q.data_ptr(), scale.data_ptr(), rows, cols, stride, q_stride, _type(out), s)
    if rc:
        _check(rc)
    return out


def _norm_inputs(x, gain, residual):
    """(columns, strides of x and of the residual)"""
    cols, x_stride = _columns(x, "x")
    _parameter(gain, cols, "gain")
    if residual is None:
        return cols, x_stride, 0
    if residual.shape != x.shape or residual.dtype is not x.dtype:
        raise ValueError("residual must have the shape and type of x")
    return cols, x_stride, _columns(residual, "residual")[1]


def rms_norm(x, gain, residual=None, eps=1e-5, out=None, *, stream=None):
    """h = x + residual (x itself without one), rounded to their type; y = h / sqrt(mean(h^2) + eps) * gain over the last dimension.
    gain: float32.  Returns (y, h, rstd), rstd float32 with x's leading dimensions.  out (for y) may be x or residual; without a residual not x,
    which is h."""
    if _torch is None:
        _load()
    if stream is not None:
        return _with_stream(stream, rms_norm, x, gain, residual, eps, out)
    kind = _type(x)
    cols, x_stride, r_stride = _norm_inputs(x, gain, residual)
    s = _stream(x, gain, residual, out)
    rstd = gain.new_empty(x.shape[:-1])
    if out is None:
        y, y_stride = _new(x), cols
    else:
        y = _like(out, x, "out")
        y_stride = _columns(y, "out")[1]
        _need(residual is not None or y.data_ptr() != x.data_ptr() or x.numel() == 0, "without a residual x is returned as h: out must be another array")
    if residual is None:
        h, h_ptr, r_ptr = x, None, None
    else:
        h = _new(x)
        h_ptr, r_ptr = h.data_ptr(), residual.data_ptr()
    rc = _lib.comp_ams_rms_norm(y.data_ptr(), h_ptr, rstd.data_ptr(), x.data_ptr(), r_ptr, gain.data_ptr(), rstd.numel(), cols, y_stride, cols, x_stride,
                                r_stride, eps, kind, s)
    if rc:
        _check(rc)
    return y, h, rstd


def rms_norm_q8(x, gain, residual=None, eps=1e-5, binary=False, *, stream=None):
    """rms_norm with y in 8 bits: returns (q int8, scale float32, h, rstd)."""
    if _torch is None:
        _load()
    if stream is not None:
        return _with_stream(stream, rms_norm_q8, x, gain, residual, eps, binary)
    kind = _type(x)
    cols, x_stride, r_stride = _norm_inputs(x, gain, residual)
    s = _stream(x, gain, residual)
    q = _new(x, _torch.int8)
    scale = gain.new_empty(x.shape[:-1])
    rstd = _torch.empty_like(scale)
    if residual is None:
        h, h_ptr, r_ptr = x, None, None
    else:
        h = _new(x)
        h_ptr, r_ptr = h.data_ptr(), residual.data_ptr()
    rc = _lib.comp_ams_rms_norm_q8(q.data_ptr(), scale.data_ptr(), h_ptr, rstd.data_ptr(), x.data_ptr(), r_ptr, gain.data_ptr(), rstd.numel(), cols, cols,
                                   cols, x_stride, r_stride, eps, 1 if binary else 0, kind, s)
    if rc:
        _check(rc)
    return q, scale, h, rstd


def rms_norm_backward(dy, h, rstd, gain, dgain, dresidual=None, scale=None, out=None, *, stream=None):
    """Backward pass of both norms from h as it was returned, or from a checkpoint of it in 8 bits (int8, with its `scale`): returns the gradient
    of x and residual alike, with dresidual, the gradient that reaches h past the norm, added to it, and writes dgain [n, cols] (a view of the
    optimiser's gradient buffer, of its type), worker w's from the w-th of n equal parts of the rows.  out may be dy, dresidual or an h of its type."""
    if _torch is None:
        _load()
    if stream is not None:
        return _with_stream(stream, rms_norm_backward, dy, h, rstd, gain, dgain, dresidual, scale, out)
    kind = _type(dy)
    cols, dy_stride = _columns(dy, "dy")
    shape = dy.shape
    lead = shape[:-1]
    if h.shape != shape:
        raise ValueError("h must have the shape of dy")
    if scale is None:
        if h.dtype is not dy.dtype:
            raise ValueError("h must have the type of dy, or be int8 with a scale")
        h_stride = _columns(h, "h")[1]
    else:
        h_stride = _bytes(h, "h")[1]
        _scales(scale, lead, "scale")
    r_stride = 0
    if dresidual is not None:
        if dresidual.shape != shape or dresidual.dtype is not dy.dtype:
            raise ValueError("dresidual must have the shape and type of dy")
        r_stride = _columns(dresidual, "dresidual")[1]
    rows = _scales(rstd, lead, "rstd")
    _parameter(gain, cols, "gain")
    g_shape, g_strides = dgain.shape, dgain.stride()
    if len(g_shape) != 2 or g_shape[1] != cols or cols > 1 and g_strides[1] != 1:
        raise ValueError(f"dgain must be [n, {cols}], dense within a worker's row")
    n = g_shape[0]
    stride = g_strides[0] if n > 1 else cols
    s = _stream(dy, h, scale, rstd, gain, dgain, dresidual, out)
    if out is None:
        dx, dx_stride = _new(dy), cols
    else:
        dx = _like(out, dy, "out")
        dx_stride = _columns(dx, "out")[1]
    work, work_ptr, work_bytes = _memory(dy, "comp_ams_rms_norm_work_bytes", rows, cols, n)
    rc = _lib.comp_ams_rms_norm_backward(dx.data_ptr(), dgain.data_ptr(), dy.data_ptr(), h.data_ptr(), _ptr(scale), rstd.data_ptr(), gain.data_ptr(),
                                         _ptr(dresidual), rows, cols, dx_stride, dy_stride, h_stride, r_stride, n, stride, kind, _type(dgain), work_ptr,
                                         work_bytes, s)
    if rc:
        _check(rc)
    return dx


def linear_q8(q, scale, weight, weight_scale, bias=None, dtype=None, out=None, *, stream=None):
    """(q @ weight.T) * scale * weight_scale + bias for q int8 [..., cols] with scale float32 of its leading dimensions and weight int8
    [outs, cols] with weight_scale float32 [outs]; bias float32 [outs] or None.  Sums are exact; the result is rounded once to `dtype` (bfloat16 if
    neither it nor out is given)."""
    if _torch is None:
        _load()
    if stream is not None:
        return _with_stream(stream, linear_q8, q, scale, weight, weight_scale, bias, dtype, out)
    cols, q_stride = _bytes(q, "q")
    w_cols, w_stride = _bytes(weight, "weight")
    w_shape = weight.shape
    if len(w_shape) != 2 or w_cols != cols:
        raise ValueError("weight must be [outs, cols]")
    lead = q.shape[:-1]
    rows, outs = _scales(scale, lead, "scale"), _scales(weight_scale, w_shape[:1], "weight_scale")
    if bias is not None:
        _parameter(bias, outs, "bias")
    s = _stream(q, scale, weight, weight_scale, bias, out)
    if out is None:
        out = q.new_empty((*lead, outs), dtype=_torch.bfloat16 if dtype is None else dtype)
        y_stride = outs
    else:
        _need(out.shape == (*lead, outs) and dtype in (None, out.dtype), "out must be [..., outs] of the type asked for")
        y_stride = _columns(out, "out")[1]
    kind = _type(out)
    work, work_ptr, work_bytes = _memory(q, "comp_ams_linear_q8_work_bytes", rows, cols, outs, _sixteens(q, q_stride), _sixteens(weight, w_stride))
    rc = _lib.comp_ams_linear_q8(out.data_ptr(), q.data_ptr(), scale.data_ptr(), weight.data_ptr(), weight_scale.data_ptr(), _ptr(bias), rows, cols, outs,
                                 y_stride, q_stride, w_stride, kind, work_ptr, work_bytes, s)
    if rc:
        _check(rc)
    return out


def linear_weight_grad(dy, q, scale, dweight, dbias=None, binary=False, *, stream=None):
    """Weight gradients of y = x @ weight.T + bias from its input in 8 bits: q int8 [..., cols] with scale, dy [..., outs].  Writes
    dweight [n, outs, cols] (or a transposed view of one that is dense as [n, cols, outs]) and dbias [n, outs], views of the optimiser's gradient
    buffer, of its type; worker w's from the w-th of n equal parts of the rows.  binary: all scales are powers of two, as
    quantize_rows(..., binary=True) gives them: of dy in 16 bits nothing is lost then, and it takes one product (bfloat16) or two (float16) in place of
    two, or of three where the gradients are fp32."""
    if _torch is None:
        _load()
    if stream is not None:
        return _with_stream(stream, linear_weight_grad, dy, q, scale, dweight, dbias, binary)
    kind = _type(dy)
    cols, q_stride = _bytes(q, "q")
    outs, dy_stride = _columns(dy, "dy")
    lead = q.shape[:-1]
    if dy.shape[:-1] != lead:
        raise ValueError("dy and q must have the same leading dimensions")
    rows = _scales(scale, lead, "scale")
    shape, strides = dweight.shape, dweight.stride()
    if len(shape) != 3 or shape[1] != outs or shape[2] != cols:
        raise ValueError(f"dweight must be [n, {outs}, {cols}]")
    n, in_first = shape[0], 0
    stride = strides[0] if n > 1 else outs * cols
    if cols and outs:
        if cols > 1 and (strides[2] != 1 or outs > 1 and strides[1] == 1):
            in_first = 1
            _need(strides[1] == 1 or outs == 1, "dweight must be dense within a worker's row")
            _need(strides[2] == outs, "dweight must be dense within a worker's row")
        else:
            _need(strides[1] == cols or outs == 1, "dweight must be dense within a worker's row")
    else:                                            # nothing of it is written
        stride = outs if dbias is None or n <= 1 or dbias.dim() != 2 else dbias.stride(0)
    if dbias is not None:
        _need(dbias.dtype is dweight.dtype and tuple(dbias.shape) == (n, outs) and (_param_grad(dbias, (outs,), "dbias") == stride or n == 1),
              "dbias must be [n, outs] with the type and worker stride of dweight")
    s = _stream(dy, q, scale, dweight, dbias)
    work, work_ptr, work_bytes = _memory(dy, "comp_ams_linear_weight_grad_work_bytes", rows, cols, outs, n, 1 if binary else 0, kind, _sixteens(dy, dy_stride))
    rc = _lib.comp_ams_linear_weight_grad(dweight.data_ptr(), _ptr(dbias), dy.data_ptr(), q.data_ptr(), scale.data_ptr(), rows, cols, outs, dy_stride,
                                          q_stride, n, stride, in_first, 1 if binary else 0, kind, _type(dweight), work_ptr, work_bytes, s)
    if rc:
        _check(rc)
