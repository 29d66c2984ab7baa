"""Refusals of the operators, without a GPU: the library answers invalid arguments before any device call, and the Python entry
points check what they are handed."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

A = 1 << 20          # an address that is aligned and never used: every call below is refused before a launch


def refused(fn, args, **change):
    args = dict(args, **change)
    rc = getattr(P.lib(), fn)(*args.values())
    return rc, P.lib().comp_ams_operators_last_error().decode()


NORM = dict(y=A, mean=A, rstd=A, x=A, gain=A, shift=A, rows=4, cols=8, x_stride=8, y_stride=8, eps=1e-5, type=0, stream=None)
NORM_BACK = dict(dx=A, dgain=A, dshift=A, dy=A, x=A, mean=A, rstd=A, gain=A, rows=4, cols=8, dx_stride=8, dy_stride=8, x_stride=8, n=2,
                 grad_stride=20, type=0, grad_type=0, work=A, work_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(y=None), dict(x=None), dict(gain=None), dict(rows=-1), dict(cols=0), dict(cols=1 << 31), dict(x_stride=7),
                                    dict(y_stride=7), dict(eps=-1.0), dict(eps=math.nan), dict(type=3), dict(type=-1), dict(x=A + 1), dict(y=A + 2),
                                    dict(gain=A + 2), dict(x_stride=1 << 60)])
def test_layer_norm_refuses(change):
    rc, text = refused("comp_ams_layer_norm", NORM, **change)
    assert rc == P.EINVAL and text.startswith("layer_norm:")


@pytest.mark.parametrize("change", [dict(dx=None), dict(dgain=None), dict(dy=None), dict(x=None), dict(mean=None), dict(gain=None), dict(n=0),
                                    dict(n=3), dict(n=70_000), dict(grad_stride=7), dict(type=5), dict(grad_type=3), dict(work=None),
                                    dict(work_bytes=4), dict(work=A + 4), dict(dx_stride=4), dict(dshift=A + 2)])
def test_layer_norm_backward_refuses(change):
    rc, text = refused("comp_ams_layer_norm_backward", NORM_BACK, **change)
    assert rc == P.EINVAL and "layer_norm" in text


def int32(*v):
    return np.array(v, dtype=np.int32)


def bias_args(at, **change):
    st = (C.c_int64 * 3)(64, 32, 8)
    args = dict(p=A, s=A, table=A, bounds=at.ctypes.data, n_buckets=at.size + 1, key_len=None, batch=2, heads=2, tq=4, tk=8,
                p_strides=st, s_strides=st, offset=0, scale=1.0, causal=0, type=0, stream=None)
    return dict(args, **change)


def test_rel_bias_softmax_refuses():
    ok = int32(-3, 0, 5)
    bad_strides = (C.c_int64 * 3)(64, 32, 7)
    for change in (dict(p=None), dict(s=None), dict(table=None), dict(bounds=None), dict(n_buckets=0), dict(n_buckets=129), dict(batch=-1),
                   dict(tk=1 << 31), dict(tq=1 << 31), dict(batch=1 << 16, heads=1 << 15), dict(offset=1 << 31), dict(offset=-(1 << 31)),
                   dict(scale=math.inf), dict(scale=math.nan), dict(type=9), dict(p_strides=None), dict(s_strides=bad_strides),
                   dict(p_strides=bad_strides), dict(s=A + 1), dict(table=A + 1), dict(key_len=A + 2)):
        rc, text = refused("comp_ams_rel_bias_softmax", bias_args(ok, **change))
        assert rc == P.EINVAL and text.startswith("rel_bias_softmax:"), change
    for bounds in (int32(1, 1), int32(2, 1), int32(-5, 0, 0)):
        rc, text = refused("comp_ams_rel_bias_softmax", bias_args(bounds))
        assert rc == P.EINVAL and "ascending" in text


def test_rel_bias_softmax_backward_refuses():
    b = int32(0)
    st = (C.c_int64 * 9)(*([64, 32, 8] * 3))
    args = dict(ds=A, dtable=A, dp=A, p=A, bounds=b.ctypes.data, n_buckets=2, key_len=None, batch=2, heads=2, tq=4, tk=8, strides=st, offset=0,
                scale=1.0, causal=0, n=2, grad_stride=4, type=1, grad_type=1, work=A, work_bytes=1 << 30, stream=None)
    for change in (dict(ds=None), dict(dtable=None), dict(dp=None), dict(p=None), dict(bounds=None), dict(n=0), dict(n=3), dict(grad_stride=3),
                   dict(grad_type=7), dict(strides=None), dict(work=None), dict(work_bytes=3), dict(heads=70_000), dict(dtable=A + 1)):
        rc, text = refused("comp_ams_rel_bias_softmax_backward", args, **change)
        assert rc == P.EINVAL and "rel_bias" in text, change


LOGP = dict(logp=A, entropy=A, idx=A, top=A, logits=A, tokens=A, rows=4, vocab=100, stride=100, k=5, type=0, work=A, work_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change", [dict(logits=None), dict(tokens=None), dict(idx=None), dict(top=None), dict(rows=-1), dict(vocab=0),
                                    dict(vocab=1 << 31), dict(stride=99), dict(k=-1), dict(k=129), dict(vocab=4, stride=4), dict(type=3), dict(logits=A + 2),
                                    dict(tokens=A + 4), dict(logp=A + 1)])
def test_token_logprobs_refuses(change):
    rc, text = refused("comp_ams_token_logprobs", LOGP, **change)
    assert rc == P.EINVAL and text.startswith("token_logprobs")


DISTILL = dict(loss=A, lse=A, logits=A, idx=A, val=A, rows=4, vocab=100, stride=100, k=5, temperature=1.0, type=0, stream=None)
BACK = dict(dlogits=A, dloss=A, logits=A, lse=A, idx=A, val=A, rows=4, vocab=100, dstride=100, stride=100, k=5, temperature=1.0, type=0, stream=None)
GRAD = dict(loss=A, dlogits=A, dloss=A, logits=A, idx=A, val=A, rows=4, vocab=100, dstride=100, stride=100, k=5, temperature=1.0, type=0, stream=None)
LISTS = [dict(logits=None), dict(idx=None), dict(val=None), dict(k=0), dict(k=129), dict(temperature=0.0), dict(temperature=-1.0),
         dict(temperature=math.nan), dict(temperature=math.inf), dict(temperature=1e-45), dict(type=4), dict(vocab=0), dict(stride=50), dict(idx=A + 1)]


@pytest.mark.parametrize("change", LISTS + [dict(loss=A + 2)])
def test_distill_refuses(change):
    assert refused("comp_ams_distill", DISTILL, **change)[0] == P.EINVAL


@pytest.mark.parametrize("change", LISTS + [dict(dlogits=None), dict(dloss=None), dict(dstride=99)])
def test_distill_gradients_refuse(change):
    assert refused("comp_ams_distill_backward", BACK, **change)[0] == P.EINVAL
    assert refused("comp_ams_distill_grad", GRAD, **change)[0] == P.EINVAL


def test_distill_backward_needs_the_statistics():
    assert refused("comp_ams_distill_backward", BACK, lse=None)[0] == P.EINVAL


def test_work_sizes_are_answered_without_a_gpu():
    n = C.c_uint64(0)
    L = P.lib()
    assert L.comp_ams_layer_norm_work_bytes(4096, 768, 8, C.byref(n)) == P.OK and n.value >= 8 * 2 * 768 * 4
    assert L.comp_ams_layer_norm_work_bytes(0, 768, 8, C.byref(n)) == P.OK
    assert L.comp_ams_layer_norm_work_bytes(4097, 768, 8, C.byref(n)) == P.EINVAL
    assert L.comp_ams_layer_norm_work_bytes(4096, 768, 8, None) == P.EINVAL
    assert L.comp_ams_rel_bias_work_bytes(2, 3, 4, 5, 32, 0, C.byref(n)) == P.OK and n.value > 0
    assert L.comp_ams_rel_bias_work_bytes(2, 3, 4, 5, 129, 0, C.byref(n)) == P.EINVAL
    assert L.comp_ams_token_logprobs_work_bytes(4, 100, 101, 0, C.byref(n)) == P.EINVAL
    assert L.comp_ams_token_logprobs_work_bytes(4, 1_000_000, 101, 0, C.byref(n)) == P.OK


def test_python_entry_points_check_what_they_are_handed():
    x, f = torch.zeros(4, 8), torch.zeros(8)
    cases = [
        lambda: P.layer_norm(x, f),                                                     # not on the GPU
        lambda: P.layer_norm(x, f[:7]), lambda: P.layer_norm(x, f.double()), lambda: P.layer_norm(x.double(), f),
        lambda: P.layer_norm(x.t(), torch.zeros(4)), lambda: P.layer_norm(torch.zeros(3, 4, 8).transpose(0, 1)[:, :2], f),
        lambda: P.layer_norm_backward(x, x[:2], f[:4], f[:4], f, x[:2, :]), lambda: P.layer_norm_backward(x, x, f[:4], f[:4], f, x[:, :7]),
        lambda: P.layer_norm_backward(x, x, f[:4], f[:4], f, x[:2], x[:3]),
        lambda: P.rel_bias_softmax(x, f, []), lambda: P.rel_bias_softmax(torch.zeros(1, 2, 3, 4), torch.zeros(3, 2), [0]),
        lambda: P.rel_bias_softmax(torch.zeros(1, 2, 3, 4), torch.zeros(2, 2), [0], key_lengths=torch.zeros(1)),
        lambda: P.rel_bias_softmax_backward(torch.zeros(1, 2, 3, 4), torch.zeros(1, 2, 3, 4), [0], torch.zeros(1, 2, 3)),
        lambda: P.token_logprobs(f), lambda: P.token_logprobs(x, torch.zeros(4)), lambda: P.token_logprobs(x),
        lambda: P.distill(x, torch.zeros(4, 2), torch.zeros(4, 2)), lambda: P.distill(x, torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)),
        lambda: P.distill_grad(x, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(3)),
        lambda: P.rel_bias_bounds(0, 5),
    ]
    for case in cases:
        with pytest.raises(ValueError):
            case()


def test_bucket_boundaries():
    for buckets in (1, 2, 3, 8, 32, 33, 128):
        for distance in (1, 2, 64, 128, 5000):
            for causal in (False, True):
                b = P.rel_bias_bounds(buckets, distance, causal)
                assert b.dtype == np.int32 and b.size == buckets - 1 and (np.diff(b) > 0).all()
                if causal and buckets > 1:
                    assert b[-1] == 0                       # one bucket for the query's own place and what lies ahead
    b = P.rel_bias_bounds(32, 128)
    assert b[0] > -128 and b[-1] < 128
    assert [int((b <= r).sum()) for r in (-1000, 1000)] == [0, 31] and len({int((b <= r).sum()) for r in range(-4, 5)}) == 9


def test_the_plain_forms_agree_with_automatic_differentiation():
    """The 64-bit forms that the kernels are compared with, checked apart from them."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(6, 11, generator=g, dtype=torch.float64, requires_grad=True)
    gain = torch.randn(11, generator=g, dtype=torch.float64, requires_grad=True)
    shift = torch.randn(11, generator=g, dtype=torch.float64, requires_grad=True)
    dy = torch.randn(6, 11, generator=g, dtype=torch.float64)
    y, mean, rstd = R.norm(x, gain, shift, 1e-5)
    want = torch.autograd.grad((y * dy).sum(), (x, gain, shift))
    got = R.norm_backward(dy, x.detach(), mean.detach(), rstd.detach(), gain.detach(), 1)
    for a, b in zip(got[:3], want):
        assert torch.allclose(a.squeeze(0) if a.shape != b.shape else a, b, rtol=1e-10, atol=1e-12)
    s = torch.randn(2, 3, 5, 7, generator=g, dtype=torch.float64, requires_grad=True)
    table = torch.randn(4, 3, generator=g, dtype=torch.float64, requires_grad=True)
    dp = torch.randn(2, 3, 5, 7, generator=g, dtype=torch.float64)
    p, _ = R.bias_softmax(s, table, [-1, 0, 3], 0.3, False, 1, [7, 4])
    want = torch.autograd.grad((p * dp).sum(), (s, table))
    got = R.bias_softmax_backward(dp, p.detach(), [-1, 0, 3], 0.3, False, 1, [7, 4], 1)
    assert torch.allclose(got[0], want[0], rtol=1e-10, atol=1e-12) and torch.allclose(got[1][0], want[1], rtol=1e-10, atol=1e-12)
    z = torch.randn(3, 20, generator=g, dtype=torch.float64, requires_grad=True)
    idx = torch.tensor([[1, 5, 19], [2, -1, 3], [-1, -1, 20]], dtype=torch.int32)
    val, w = torch.randn(3, 3, generator=g), torch.rand(3, generator=g)
    out = R.distill(z, idx, val, 2.0, w)
    want = torch.autograd.grad((out[0] * w).sum(), z)[0]
    assert torch.allclose(out[2].detach(), want, rtol=1e-9, atol=1e-12)
