"""Operators of language-model training next to the compressed optimiser (include/comp_ams_operators.h): layer norm, the
softmax of scores with a learned relative position bias, token log probabilities, and distillation from a teacher's top
logits.  Tensors are torch CUDA(HIP) tensors; the calls are asynchronous on torch's current stream, or on the raw hipStream_t
that every one of them takes as `stream=`, and do not synchronise.

Parameters are fp32 tensors, as a rule views of the flat model.  Parameter gradients are tensors whose first dimension is the
worker, as a rule views of the gradient buffer [n, d] that CompAms.step takes:

    gain, shift = theta[a:a + c], theta[a + c:a + 2 * c]
    y, mean, rstd = layer_norm(x, gain, shift)
    dx = layer_norm_backward(dy, x, mean, rstd, gain, grads[:, a:a + c], grads[:, a + c:a + 2 * c])

No graph is recorded for automatic differentiation: results do not require a gradient, also where inputs do, and each
backward pass is a call of its own.

Arguments that the library would not take raise ValueError before anything is launched; what the library itself refuses
raises CompAmsError.
"""
from __future__ import annotations

import ctypes as C
import functools

import numpy as np

from .binding import OK, CompAmsError, lib

_TYPES = {}


def _type(t):
    if not _TYPES:
        import torch
        _TYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise ValueError(f"float32, bfloat16 or float16 is needed, not {t.dtype}") from None


def _check(rc):
    if rc:
        raise CompAmsError(rc, lib().comp_ams_operators_last_error().decode())


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _on_stream(fn):
    """With a raw stream given, the call runs with that stream as torch's current one, so that what it allocates belongs to it:
    memory of another stream may still be in use there."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        import torch
        with torch.cuda.stream(torch.cuda.ExternalStream(stream)):
            return fn(*args, **kw)
    return call


def _stream(like, *tensors):
    """The raw current stream; all tensors must be on the GPU of `like`, which has to be the current one."""
    import torch
    if not like.is_cuda:
        raise ValueError("tensors must be on the GPU")
    dev = like.get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("all tensors must be on the same GPU")
    if dev != torch.cuda.current_device():
        raise ValueError(f"the tensors are on GPU {dev}, which is not the current one")
    return torch._C._cuda_getCurrentRawStream(dev)      # what torch.cuda.current_stream(dev).cuda_stream gives, without building a Stream


def _rows(t, what):
    """(rows, columns, row stride) of a tensor [..., columns] whose rows are evenly spaced and dense."""
    shape = t.shape
    _need(len(shape) >= 1, f"{what} needs at least one dimension")
    cols = shape[-1]
    if t.is_contiguous():
        return (t.numel() // cols if cols else 0), cols, max(cols, 1)
    _need(t.stride(-1) == 1 or cols <= 1, f"the last dimension of {what} must be dense")
    if t.dim() == 1:
        return 1, cols, cols
    if t.dim() == 2:
        return t.shape[0], cols, t.stride(0) if t.shape[0] > 1 else max(cols, 1)
    rows, stride, span = 1, None, None
    for size, st in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride, span = st, size * st
        else:
            _need(st == span or rows == 0, f"the rows of {what} must be evenly spaced")
            span = size * st
        rows *= size
    return rows, cols, max(cols, 1) if stride is None else stride


def _vector(t, size, dtype, what):
    _need(t.dtype == dtype and t.is_contiguous() and t.numel() == size, f"{what} must be a dense {dtype} tensor of {size} elements")


def _like(out, t, what):
    """out (new and dense if None), which must have t's shape and type."""
    import torch
    if out is None:
        return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)
    _need(out.shape == t.shape and out.dtype == t.dtype, f"{what} must have the shape and type of its input")
    return out


@functools.lru_cache(maxsize=4096)
def _work_bytes(name, *args):
    need = C.c_uint64(0)
    _check(getattr(lib(), name)(*args, C.byref(need)))
    return need.value


def _work(name, device, *args):
    """(work tensor or None, pointer, bytes) for the size that the library asks for."""
    need = _work_bytes(name, *args)
    if need == 0:
        return None, None, 0
    import torch
    w = torch.empty(need, dtype=torch.uint8, device=device)
    return w, w.data_ptr(), need


def _param_grad(t, shape, what):
    """Worker stride of a parameter gradient [n, *shape] that is dense within a worker."""
    _need(t.dim() == len(shape) + 1 and tuple(t.shape[1:]) == shape, f"{what} must be [n, {', '.join(map(str, shape))}]")
    dense = 1
    for size, st in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        _need(st == dense or size <= 1, f"{what} must be dense within a worker's row")
        dense *= size
    return t.stride(0) if t.shape[0] > 1 else dense


@_on_stream
def layer_norm(x, gain, shift=None, eps=1e-5, out=None):
    """y = (x - mean) / sqrt(var + eps) * gain + shift over the last dimension of x (float32, bfloat16 or float16).
    gain, shift: float32.  Returns (y, mean, rstd), mean and rstd float32 with x's leading dimensions.  out may be x."""
    import torch
    rows, cols, x_stride = _rows(x, "x")
    _vector(gain, cols, torch.float32, "gain")
    if shift is not None:
        _vector(shift, cols, torch.float32, "shift")
    s = _stream(x, gain, shift, out)
    y = _like(out, x, "out")
    y_stride = x_stride if out is None and x.is_contiguous() else _rows(y, "out")[2]
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    _check(lib().comp_ams_layer_norm(y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), x.data_ptr(), gain.data_ptr(),
                                     None if shift is None else shift.data_ptr(), rows, cols, x_stride, y_stride, eps, _type(x), s))
    return y, mean, rstd


@_on_stream
def layer_norm_backward(dy, x, mean, rstd, gain, dgain, dshift=None, out=None):
    """Backward pass of layer_norm: returns dx and writes the parameter gradients, dgain [n, cols] and dshift [n, cols]
    (views of the optimiser's gradient buffer, of its type), worker w's from the w-th of n equal parts of the rows.
    out may be dy or x."""
    import torch
    rows, cols, x_stride = _rows(x, "x")
    _need(dy.shape == x.shape and dy.dtype == x.dtype, "dy must have the shape and type of x")
    _, _, dy_stride = _rows(dy, "dy")
    _vector(mean, rows, torch.float32, "mean")
    _vector(rstd, rows, torch.float32, "rstd")
    _vector(gain, cols, torch.float32, "gain")
    stride = _param_grad(dgain, (cols,), "dgain")
    n = dgain.shape[0]
    if dshift is not None:
        _need(dshift.dtype == dgain.dtype and dshift.shape == dgain.shape and (_param_grad(dshift, (cols,), "dshift") == stride or n == 1),
              "dshift must have the shape, type and stride of dgain")
    s = _stream(x, dy, mean, rstd, gain, dgain, dshift, out)
    dx = _like(out, x, "out")
    _, _, dx_stride = _rows(dx, "out")
    L = lib()
    work, work_ptr, work_bytes = _work("comp_ams_layer_norm_work_bytes", x.device, rows, cols, n)
    _check(L.comp_ams_layer_norm_backward(dx.data_ptr(), dgain.data_ptr(), None if dshift is None else dshift.data_ptr(), dy.data_ptr(),
                                          x.data_ptr(), mean.data_ptr(), rstd.data_ptr(), gain.data_ptr(), rows, cols, dx_stride,
                                          dy_stride, x_stride, n, stride, _type(x), _type(dgain), work_ptr, work_bytes, s))
    return dx


def rel_bias_bounds(buckets, distance, causal=False):
    """Bucket boundaries for rel_bias_softmax: int32 array of buckets - 1 ascending relative positions (key minus query).
    On either side of a query (with causal on the side of the past alone, one bucket for everything ahead) half of the
    buckets hold one position each and the others grow with the distance, the last one from below `distance` on."""
    _need(buckets >= 1 and distance >= 1, "buckets and distance must be at least 1")

    def widening(many):
        near = (many + 1) // 2
        at = list(range(1, near + 1))
        for q in range(1, many - near + 1):
            at.append(max(at[-1] + 1, int(near * (distance / near) ** (q / (many - near + 1)))))
        return at

    left = buckets - 1 if causal else (buckets - 1) // 2
    past = [1 - at for at in reversed(widening(left))]
    return np.array(past + widening(buckets - 1 - left), dtype=np.int32)


def _bounds(bounds):
    if type(bounds) is np.ndarray and bounds.dtype == np.int32 and bounds.flags.c_contiguous:
        b = bounds
    else:
        b = np.asarray(bounds)
        if b.size:
            _need(b.dtype.kind in "iuf" and np.isfinite(b).all() and (b == np.floor(b)).all() and -2 ** 31 <= b.min() and b.max() < 2 ** 31,
                  "bounds must be whole numbers of 32 bits")
        b = np.ascontiguousarray(b, dtype=np.int32)
    _need(b.ndim == 1, "bounds must be one-dimensional")
    return b


def _scores(t, what):
    _need(t.dim() == 4, f"{what} must be [batch, heads, queries, keys]")
    _need(t.stride(3) == 1 or t.shape[3] <= 1, f"the last dimension of {what} must be dense")
    return t.stride()[:3]


def _lengths(key_lengths, batch):
    import torch
    if key_lengths is not None:
        _vector(key_lengths, batch, torch.int32, "key_lengths")
    return None if key_lengths is None else key_lengths.data_ptr()


@_on_stream
def rel_bias_softmax(scores, table, bounds, scale=1.0, causal=False, offset=0, key_lengths=None, out=None):
    """Softmax over the keys of scale * scores + table[bucket(key - query - offset), head].

    scores [batch, heads, queries, keys] with a dense last dimension; table float32 [buckets, heads] dense; bounds:
    buckets - 1 ascending relative positions (an int32 array; see rel_bias_bounds), the bucket of r being how many of them are <= r.
    A query sees the first key_lengths[batch] keys (int32) and, with causal, those at relative positions <= 0; offset is the
    position of the first query among the keys.  A query that sees nothing gets zeros.  out may be scores."""
    import torch
    s_strides = _scores(scores, "scores")
    batch, heads, tq, tk = scores.shape
    b = _bounds(bounds)
    _vector(table, (b.size + 1) * heads, torch.float32, "table")
    _need(tuple(table.shape) == (b.size + 1, heads), "table must be [buckets, heads] with one bucket more than there are bounds")
    st = _stream(scores, table, key_lengths, out)
    p = _like(out, scores, "out")
    p_strides = _scores(p, "out")
    _check(lib().comp_ams_rel_bias_softmax(p.data_ptr(), scores.data_ptr(), table.data_ptr(), b.ctypes.data, b.size + 1,
                                           _lengths(key_lengths, batch), batch, heads, tq, tk, (C.c_int64 * 3)(*p_strides),
                                           (C.c_int64 * 3)(*s_strides), offset, scale, 1 if causal else 0, _type(scores), st))
    return p


@_on_stream
def rel_bias_softmax_backward(dprobs, probs, bounds, dtable, scale=1.0, causal=False, offset=0, key_lengths=None, out=None):
    """Backward pass of rel_bias_softmax from the probabilities it returned: returns the gradient of the scores and writes
    dtable [n, buckets, heads] (a view of the optimiser's gradient buffer, of its type), worker w's from the w-th of n equal parts
    of the batch.  Keys of probability zero take no gradient.  out may be dprobs."""
    dp_strides, p_strides = _scores(dprobs, "dprobs"), _scores(probs, "probs")
    _need(dprobs.shape == probs.shape and dprobs.dtype == probs.dtype, "dprobs must have the shape and type of probs")
    batch, heads, tq, tk = probs.shape
    b = _bounds(bounds)
    stride = _param_grad(dtable, (b.size + 1, heads), "dtable")
    st = _stream(probs, dprobs, dtable, key_lengths, out)
    ds = _like(out, dprobs, "out")
    ds_strides = _scores(ds, "out")
    L, kind = lib(), _type(probs)
    work, work_ptr, work_bytes = _work("comp_ams_rel_bias_work_bytes", probs.device, batch, heads, tq, tk, b.size + 1, kind)
    _check(L.comp_ams_rel_bias_softmax_backward(ds.data_ptr(), dtable.data_ptr(), dprobs.data_ptr(), probs.data_ptr(), b.ctypes.data,
                                                b.size + 1, _lengths(key_lengths, batch), batch, heads, tq, tk,
                                                (C.c_int64 * 9)(*ds_strides, *dp_strides, *p_strides), offset, scale, 1 if causal else 0,
                                                dtable.shape[0], stride, kind, _type(dtable), work_ptr, work_bytes, st))
    return ds


@_on_stream
def token_logprobs(logits, tokens=None, k=0):
    """Under logits [rows, vocab]: (log probabilities of `tokens` [rows] int64 or None, entropies [rows], the k best tokens
    [rows, k] int32 - largest first, the lower token first among equals - and their log probabilities [rows, k]), float32."""
    import torch
    _need(logits.dim() == 2, "logits must be [rows, vocab]")
    rows, vocab, stride = _rows(logits, "logits")
    if tokens is not None:
        _vector(tokens, rows, torch.int64, "tokens")
    s = _stream(logits, tokens)
    L, kind = lib(), _type(logits)
    work, work_ptr, work_bytes = _work("comp_ams_token_logprobs_work_bytes", logits.device, rows, vocab, k, kind)      # looks at k
    f32 = dict(dtype=torch.float32, device=logits.device)
    logp = None if tokens is None else torch.empty(rows, **f32)
    entropy = torch.empty(rows, **f32) if logp is None else torch.empty_like(logp)
    top = torch.empty((rows, k), **f32)
    idx = torch.empty_like(top, dtype=torch.int32)
    _check(L.comp_ams_token_logprobs(None if logp is None else logp.data_ptr(), entropy.data_ptr(), idx.data_ptr(), top.data_ptr(),
                                     logits.data_ptr(), None if tokens is None else tokens.data_ptr(), rows, vocab, stride, k, kind,
                                     work_ptr, work_bytes, s))
    return logp, entropy, idx, top


def _teacher(logits, idx, val):
    import torch
    _need(logits.dim() == 2, "logits must be [rows, vocab]")
    rows, vocab, stride = _rows(logits, "logits")
    _need(idx.dim() == 2 and idx.shape[0] == rows and idx.shape == val.shape, "idx and val must be [rows, k]")
    _need(idx.dtype == torch.int32 and val.dtype == torch.float32 and idx.is_contiguous() and val.is_contiguous(),
          "idx must be int32, val float32, both dense")
    return rows, vocab, stride, idx.shape[1]


@_on_stream
def distill(logits, idx, val, temperature=1.0):
    """Distillation loss of logits [rows, vocab] against a teacher's top lists: idx int32 [rows, k] (tokens; entries outside the
    vocabulary are not there) and val float32 [rows, k] (its logits or log probabilities).  Returns (loss [rows], lse [rows]): T^2 KL of
    the teacher's distribution over its list from the student's over the vocabulary, both at temperature T."""
    import torch
    rows, vocab, stride, k = _teacher(logits, idx, val)
    s = _stream(logits, idx, val)
    loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
    lse = torch.empty_like(loss)
    _check(lib().comp_ams_distill(loss.data_ptr(), lse.data_ptr(), logits.data_ptr(), idx.data_ptr(), val.data_ptr(), rows, vocab, stride,
                                  k, temperature, _type(logits), s))
    return loss, lse


@_on_stream
def distill_backward(dloss, logits, lse, idx, val, temperature=1.0, out=None):
    """Gradient of the logits from the gradients dloss [rows] of distill's losses and the lse it returned, whose rounding to float32 the
    probabilities carry: for rows of very large logits use distill_grad.  out may be logits."""
    import torch
    rows, vocab, stride, k = _teacher(logits, idx, val)
    _vector(dloss, rows, torch.float32, "dloss")
    _vector(lse, rows, torch.float32, "lse")
    s = _stream(logits, dloss, lse, idx, val, out)
    d = _like(out, logits, "out")
    _check(lib().comp_ams_distill_backward(d.data_ptr(), dloss.data_ptr(), logits.data_ptr(), lse.data_ptr(), idx.data_ptr(), val.data_ptr(),
                                           rows, vocab, _rows(d, "out")[2], stride, k, temperature, _type(logits), s))
    return d


@_on_stream
def distill_grad(logits, idx, val, dloss, temperature=1.0, out=None):
    """distill and distill_backward in one pass over the logits, for a loss whose weights dloss [rows] are known beforehand.
    Returns (loss [rows], gradient of the logits).  out may be logits."""
    import torch
    rows, vocab, stride, k = _teacher(logits, idx, val)
    _vector(dloss, rows, torch.float32, "dloss")
    s = _stream(logits, dloss, idx, val, out)
    d = _like(out, logits, "out")
    loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
    _check(lib().comp_ams_distill_grad(loss.data_ptr(), d.data_ptr(), dloss.data_ptr(), logits.data_ptr(), idx.data_ptr(), val.data_ptr(),
                                       rows, vocab, _rows(d, "out")[2], stride, k, temperature, _type(logits), s))
    return loss, d
