"""Operators on rows held in 8 bits (include/comp_ams_rows8.h): the root-mean-square norm with the residual's addition and an output in
8 bits, activation checkpoints in 8 bits, weight gradients formed from them per worker, and the product of 8-bit integers with a scale for
each token and channel.  Conventions are those of operators.py.

A row in 8 bits is q (int8) and one float32 scale: q = rint(x / scale), scale = absmax / 127, or with binary=True the least power of two
not below that, which makes q * scale exact in every type.

    q, scale, h, rstd = rms_norm_q8(x, gain, residual, binary=True)         # 8 bits for the product, and kept for the backward pass
    y = linear_q8(q, scale, wq, wscale)                                     # wq, wscale = quantize_rows(weight)
    linear_weight_grad(dy, q, scale, grads[:, a:b].unflatten(1, (outs, cols)), binary=True)
    dx = rms_norm_backward(dx_product, h, rstd, gain, grads[:, c:c + cols], dresidual=dh)
"""
from __future__ import annotations

from .binding import lib
from .operators import _check, _like, _need, _on_stream, _param_grad, _rows, _stream, _type, _vector, _work


def _bytes(t, what):
    """_rows of an int8 tensor."""
    import torch
    if t.dtype != torch.int8:
        raise ValueError(f"{what} must be int8")
    return _rows(t, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _scales(t, like, what):
    """A dense float32 tensor with one number for each row of `like`; how many."""
    import torch
    if t.shape != like.shape[:-1] or t.dtype != torch.float32 or not t.is_contiguous():
        raise ValueError(f"{what} must be a dense float32 tensor with one number for each row")
    return t.numel()


def _new(t, dtype=None):
    """A dense tensor of t's shape (empty_like where t is dense: half the time of empty)."""
    import torch
    if t.is_contiguous():
        return torch.empty_like(t) if dtype is None else torch.empty_like(t, dtype=dtype)
    return t.new_empty(t.shape, dtype=dtype)


def _sixteens(t, stride):
    """Whether an int8 or 16-bit array is known to have its rows at multiples of 16 bytes."""
    return 1 if (t.data_ptr() | stride * t.element_size()) % 16 == 0 and stride < 1 << 22 else 0


@_on_stream
def quantize_rows(x, binary=False):
    """x [..., cols] (float32, bfloat16 or float16) in 8 bits: (q int8 of its shape, scale float32 of its leading dimensions).  A row with a
    NaN or an infinity has the scale NaN."""
    import torch
    kind = _type(x)
    _, cols, x_stride = _rows(x, "x")
    s = _stream(x)
    q = _new(x, torch.int8)
    scale = x.new_empty(x.shape[:-1], dtype=torch.float32)
    _check(lib().comp_ams_quantize_rows(q.data_ptr(), scale.data_ptr(), x.data_ptr(), scale.numel(), cols, cols, x_stride, 1 if binary else 0, kind, s))
    return q, scale


@_on_stream
def restore_rows(q, scale, dtype=None, out=None):
    """q * scale in `dtype` (float32 if neither it nor out is given), rounded once."""
    import torch
    _, cols, q_stride = _bytes(q, "q")
    rows = _scales(scale, q, "scale")
    s = _stream(q, scale, out)
    if out is None:
        out = _new(q, torch.float32 if dtype is None else dtype)
        stride = cols
    else:
        _need(out.shape == q.shape and dtype in (None, out.dtype), "out must have the shape of q and the type asked for")
        stride = _rows(out, "out")[2]
    _check(lib().comp_ams_restore_rows(out.data_ptr(), q.data_ptr(), scale.data_ptr(), rows, cols, stride, q_stride, _type(out), s))
    return out


def _norm_inputs(x, gain, residual):
    """(rows, columns, strides of x and of the residual)"""
    import torch
    rows, cols, x_stride = _rows(x, "x")
    if gain.dtype != torch.float32 or gain.numel() != cols or not gain.is_contiguous():
        raise ValueError(f"gain must be a dense float32 tensor of {cols} elements")
    if residual is None:
        return rows, cols, x_stride, 0
    _need(residual.shape == x.shape and residual.dtype == x.dtype, "residual must have the shape and type of x")
    return rows, cols, x_stride, _rows(residual, "residual")[2]


@_on_stream
def rms_norm(x, gain, residual=None, eps=1e-5, out=None):
    """h = x + residual (x itself without one), rounded to their type; y = h / sqrt(mean(h^2) + eps) * gain over the last dimension.
    gain: float32.  Returns (y, h, rstd), rstd float32 with x's leading dimensions.  out (for y) may be x or residual; without a residual not x,
    which is h."""
    kind = _type(x)
    rows, cols, x_stride, r_stride = _norm_inputs(x, gain, residual)
    s = _stream(x, gain, residual, out)
    if out is None:
        y, y_stride = _new(x), cols
    else:
        y = _like(out, x, "out")
        y_stride = _rows(y, "out")[2]
        _need(residual is not None or y.data_ptr() != x.data_ptr() or rows == 0, "without a residual x is returned as h: out must be another array")
    h = x if residual is None else _new(x)
    rstd = gain.new_empty(x.shape[:-1])
    _check(lib().comp_ams_rms_norm(y.data_ptr(), None if residual is None else h.data_ptr(), rstd.data_ptr(), x.data_ptr(), _ptr(residual),
                                   gain.data_ptr(), rows, cols, y_stride, cols, x_stride, r_stride, eps, kind, s))
    return y, h, rstd


@_on_stream
def rms_norm_q8(x, gain, residual=None, eps=1e-5, binary=False):
    """rms_norm with y in 8 bits: returns (q int8, scale float32, h, rstd)."""
    import torch
    kind = _type(x)
    rows, cols, x_stride, r_stride = _norm_inputs(x, gain, residual)
    s = _stream(x, gain, residual)
    h = x if residual is None else _new(x)
    q = _new(x, torch.int8)
    scale = gain.new_empty(x.shape[:-1])
    rstd = torch.empty_like(scale)
    _check(lib().comp_ams_rms_norm_q8(q.data_ptr(), scale.data_ptr(), None if residual is None else h.data_ptr(), rstd.data_ptr(), x.data_ptr(),
                                      _ptr(residual), gain.data_ptr(), rows, cols, cols, cols, x_stride, r_stride, eps, 1 if binary else 0, kind, s))
    return q, scale, h, rstd


@_on_stream
def rms_norm_backward(dy, h, rstd, gain, dgain, dresidual=None, scale=None, out=None):
    """Backward pass of both norms from h as it was returned, or from a checkpoint of it in 8 bits (int8, with its `scale`): returns the gradient
    of x and residual alike, with dresidual, the gradient that reaches h past the norm, added to it, and writes dgain [n, cols] (a view of the
    optimiser's gradient buffer, of its type), worker w's from the w-th of n equal parts of the rows.  out may be dy, dresidual or an h of its type."""
    import torch
    kind = _type(dy)
    rows, cols, dy_stride = _rows(dy, "dy")
    _need(h.shape == dy.shape, "h must have the shape of dy")
    if scale is None:
        _need(h.dtype == dy.dtype, "h must have the type of dy, or be int8 with a scale")
        h_stride = _rows(h, "h")[2]
    else:
        h_stride = _bytes(h, "h")[2]
        _scales(scale, dy, "scale")
    r_stride = 0
    if dresidual is not None:
        _need(dresidual.shape == dy.shape and dresidual.dtype == dy.dtype, "dresidual must have the shape and type of dy")
        r_stride = _rows(dresidual, "dresidual")[2]
    _scales(rstd, dy, "rstd")
    _vector(gain, cols, torch.float32, "gain")
    stride, n = _param_grad(dgain, (cols,), "dgain"), dgain.shape[0]
    s = _stream(dy, h, scale, rstd, gain, dgain, dresidual, out)
    if out is None:
        dx, dx_stride = _new(dy), cols
    else:
        dx = _like(out, dy, "out")
        dx_stride = _rows(dx, "out")[2]
    work, work_ptr, work_bytes = _work("comp_ams_rms_norm_work_bytes", dy.device, rows, cols, n)
    _check(lib().comp_ams_rms_norm_backward(dx.data_ptr(), dgain.data_ptr(), dy.data_ptr(), h.data_ptr(), _ptr(scale), rstd.data_ptr(), gain.data_ptr(),
                                            _ptr(dresidual), rows, cols, dx_stride, dy_stride, h_stride, r_stride, n, stride, kind, _type(dgain),
                                            work_ptr, work_bytes, s))
    return dx


@_on_stream
def linear_q8(q, scale, weight, weight_scale, bias=None, dtype=None, out=None):
    """(q @ weight.T) * scale * weight_scale + bias for q int8 [..., cols] with scale float32 of its leading dimensions and weight int8
    [outs, cols] with weight_scale float32 [outs]; bias float32 [outs] or None.  Sums are exact; the result is rounded once to `dtype` (bfloat16 if
    neither it nor out is given)."""
    import torch
    _, cols, q_stride = _bytes(q, "q")
    _need(weight.dim() == 2 and weight.shape[1] == cols, "weight must be [outs, cols]")
    w_stride = _bytes(weight, "weight")[2]
    rows, outs = _scales(scale, q, "scale"), _scales(weight_scale, weight, "weight_scale")
    if bias is not None:
        _vector(bias, outs, torch.float32, "bias")
    s = _stream(q, scale, weight, weight_scale, bias, out)
    if out is None:
        out = q.new_empty((*q.shape[:-1], outs), dtype=torch.bfloat16 if dtype is None else dtype)
        y_stride = outs
    else:
        _need(out.shape == (*q.shape[:-1], outs) and dtype in (None, out.dtype), "out must be [..., outs] of the type asked for")
        y_stride = _rows(out, "out")[2]
    kind = _type(out)
    work, work_ptr, work_bytes = _work("comp_ams_linear_q8_work_bytes", q.device, rows, cols, outs, _sixteens(q, q_stride), _sixteens(weight, w_stride))
    _check(lib().comp_ams_linear_q8(out.data_ptr(), q.data_ptr(), scale.data_ptr(), weight.data_ptr(), weight_scale.data_ptr(), _ptr(bias), rows, cols,
                                    outs, y_stride, q_stride, w_stride, kind, work_ptr, work_bytes, s))
    return out


@_on_stream
def linear_weight_grad(dy, q, scale, dweight, dbias=None, binary=False):
    """Weight gradients of y = x @ weight.T + bias from its input in 8 bits: q int8 [..., cols] with scale, dy [..., outs].  Writes
    dweight [n, outs, cols] (or a transposed view of one that is dense as [n, cols, outs]) and dbias [n, outs], views of the optimiser's gradient
    buffer, of its type; worker w's from the w-th of n equal parts of the rows.  binary: all scales are powers of two, as
    quantize_rows(..., binary=True) gives them: bfloat16 gradients then take half the products."""
    kind = _type(dy)
    _, cols, q_stride = _bytes(q, "q")
    _need(dy.dim() >= 1 and dy.shape[:-1] == q.shape[:-1], "dy and q must have the same leading dimensions")
    _, outs, dy_stride = _rows(dy, "dy")
    rows = _scales(scale, q, "scale")
    if dweight.dim() != 3 or tuple(dweight.shape[1:]) != (outs, cols):
        raise ValueError(f"dweight must be [n, {outs}, {cols}]")
    n = dweight.shape[0]
    if cols and outs:
        in_first = dweight.stride(2) != 1 and cols > 1 or dweight.stride(1) == 1 and outs > 1 and cols > 1
        stride = _param_grad(dweight.transpose(1, 2) if in_first else dweight, (cols, outs) if in_first else (outs, cols), "dweight")
    else:
        in_first, stride = False, max(dweight.stride(0), outs)           # nothing of it is written
    if dbias is not None:
        _need(dbias.dtype == dweight.dtype and tuple(dbias.shape) == (n, outs) and (_param_grad(dbias, (outs,), "dbias") == stride or n == 1),
              "dbias must be [n, outs] with the type and worker stride of dweight")
    s = _stream(dy, q, scale, dweight, dbias)
    work, work_ptr, work_bytes = _work("comp_ams_linear_weight_grad_work_bytes", dy.device, rows, cols, outs, n, 1 if binary else 0, kind,
                                       _sixteens(dy, dy_stride))
    _check(lib().comp_ams_linear_weight_grad(dweight.data_ptr(), _ptr(dbias), dy.data_ptr(), q.data_ptr(), scale.data_ptr(), rows, cols, outs, dy_stride,
                                             q_stride, n, stride, 1 if in_first else 0, 1 if binary else 0, kind, _type(dweight), work_ptr, work_bytes, s))
