"""Refusals of the operators on rows in 8 bits, without a GPU: the library answers invalid arguments before any device call, and the
Python entry points check what they are handed."""
import ctypes as C
import math

import pytest
import torch

import paper_2111_00705_amd as P

A = 1 << 20          # an address that is aligned and never used: every call below is refused before a launch
B31 = 1 << 31


def refused(fn, args, **change):
    args = dict(args, **change)
    rc = getattr(P.lib(), fn)(*args.values())
    return rc, P.lib().comp_ams_operators_last_error().decode()


QUANT = dict(q=A, scale=A, x=A, rows=4, cols=8, q_stride=8, x_stride=8, binary=0, type=0, stream=None)
RESTORE = dict(x=A, q=A, scale=A, rows=4, cols=8, x_stride=8, q_stride=8, type=0, stream=None)
NORM = dict(y=A, h=A + 64, rstd=A, x=A, residual=A, gain=A, rows=4, cols=8, y_stride=8, h_stride=8, x_stride=8, r_stride=8, eps=1e-5, type=0, stream=None)
NORM8 = dict(q=A, scale=A, h=A, rstd=A, x=A, residual=A, gain=A, rows=4, cols=8, q_stride=8, h_stride=8, x_stride=8, r_stride=8, eps=1e-5, binary=0, type=0,
             stream=None)
BACK = dict(dx=A, dgain=A, dy=A, h=A, h_scale=None, rstd=A, gain=A, dresidual=A, rows=4, cols=8, dx_stride=8, dy_stride=8, h_stride=8, r_stride=8, n=2,
            grad_stride=20, type=0, grad_type=0, work=A, work_bytes=1 << 30, stream=None)
LINEAR = dict(y=A, q=A, scale=A, w=A, w_scale=A, bias=A, rows=4, cols=8, outs=6, y_stride=6, q_stride=8, w_stride=8, type=0, work=None, work_bytes=0, stream=None)
WEIGHT = dict(dweight=A, dbias=A, dy=A, q=A, scale=A, rows=4, cols=8, outs=6, dy_stride=6, q_stride=8, n=2, grad_stride=60, in_first=0, binary=0, type=0,
              grad_type=0, work=A, work_bytes=1 << 30, stream=None)

CALLS = [
    ("quantize_rows", QUANT, [dict(q=None), dict(scale=None), dict(x=None), dict(rows=-1), dict(rows=B31), dict(cols=-1), dict(cols=B31), dict(q_stride=7),
                              dict(x_stride=7), dict(type=3), dict(type=-1), dict(x=A + 2), dict(scale=A + 2), dict(q_stride=1 << 60)]),
    ("restore_rows", RESTORE, [dict(q=None), dict(scale=None), dict(x=None), dict(rows=-1), dict(cols=B31), dict(q_stride=7), dict(x_stride=7), dict(type=3),
                               dict(x=A + 1), dict(scale=A + 1)]),
    ("rms_norm", NORM, [dict(y=None), dict(x=None), dict(gain=None), dict(rows=-1), dict(rows=1 << 40), dict(cols=0), dict(cols=B31), dict(x_stride=7),
                        dict(y_stride=7), dict(h_stride=7), dict(r_stride=7), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(type=3), dict(x=A + 1),
                        dict(residual=A + 2), dict(h=A + 2), dict(gain=A + 2), dict(rstd=A + 1), dict(h=A), dict(x_stride=1 << 60)]),
    ("rms_norm_q8", NORM8, [dict(q=None), dict(scale=None), dict(x=None), dict(gain=None), dict(cols=0), dict(q_stride=7), dict(h_stride=7), dict(eps=-1.0),
                            dict(type=9), dict(scale=A + 2)]),
    ("rms_norm_backward", BACK, [dict(dx=None), dict(dgain=None), dict(dy=None), dict(h=None), dict(rstd=None), dict(gain=None), dict(n=0), dict(n=3),
                                 dict(n=70_000), dict(grad_stride=7), dict(type=5), dict(grad_type=3), dict(work=None), dict(work_bytes=4), dict(work=A + 4),
                                 dict(dx_stride=4), dict(dy_stride=4), dict(h_stride=4), dict(r_stride=4), dict(dresidual=A + 2), dict(h=A + 1),
                                 dict(h_scale=A + 2), dict(h_scale=A, h_stride=7)]),
    ("linear_q8", LINEAR, [dict(y=None), dict(q=None), dict(scale=None), dict(w=None), dict(w_scale=None), dict(rows=-1), dict(rows=B31), dict(cols=-1),
                           dict(cols=131_072), dict(outs=-1), dict(outs=B31), dict(y_stride=5), dict(q_stride=7), dict(w_stride=7), dict(type=3), dict(y=A + 2),
                           dict(bias=A + 2), dict(scale=A + 1), dict(w_scale=A + 2), dict(rows=B31 - 1, outs=B31 - 1, y_stride=1 << 29),
                           dict(rows=100, cols=4096, outs=100, q_stride=4096, w_stride=4096, y_stride=100), dict(rows=100, cols=9, q_stride=9, w_stride=9)]),
    ("linear_weight_grad", WEIGHT, [dict(dweight=None), dict(dy=None), dict(q=None), dict(scale=None), dict(rows=-2), dict(rows=5), dict(n=0), dict(n=70_000),
                                    dict(cols=-1), dict(cols=B31), dict(outs=B31), dict(cols=1 << 21, outs=1 << 20), dict(dy_stride=5), dict(q_stride=7),
                                    dict(grad_stride=47), dict(type=3), dict(grad_type=-1), dict(work=None), dict(work_bytes=8), dict(work=A + 8),
                                    dict(dy=A + 1), dict(dweight=A + 1), dict(dbias=A + 2), dict(scale=A + 2), dict(rows=1 << 40)]),
]


@pytest.mark.parametrize("name,args,change", [(n, a, c) for n, a, cs in CALLS for c in cs], ids=lambda v: str(v) if not isinstance(v, dict) or len(v) < 5 else "")
def test_the_library_refuses(name, args, change):
    rc, text = refused("comp_ams_" + name, args, **change)
    assert rc == P.EINVAL and text.startswith(name), text


def test_nothing_to_do_is_no_error():
    for name, args, change in (("quantize_rows", QUANT, dict(rows=0, q=None, x=None, scale=None)), ("restore_rows", RESTORE, dict(cols=0, q=None, x=None)),
                               ("rms_norm", NORM, dict(rows=0, x=None, y=None, h=None, residual=None)), ("rms_norm_q8", NORM8, dict(rows=0, q=None, scale=None)),
                               ("linear_q8", LINEAR, dict(rows=0, y=None, q=None, scale=None)), ("linear_q8", LINEAR, dict(outs=0, y=None, w=None, w_scale=None)),
                               ("linear_weight_grad", WEIGHT, dict(outs=0, dbias=None, dweight=None))):
        rc, text = refused("comp_ams_" + name, args, **change)
        assert rc == P.OK, text


def test_work_bytes():
    L, n = P.lib(), C.c_uint64(99)
    assert L.comp_ams_rms_norm_work_bytes(4096, 768, 8, C.byref(n)) == P.OK and n.value >= 8 * 768 * 4
    assert L.comp_ams_rms_norm_work_bytes(4097, 768, 8, C.byref(n)) == P.EINVAL and L.comp_ams_rms_norm_work_bytes(4096, 768, 8, None) == P.EINVAL
    assert L.comp_ams_linear_q8_work_bytes(4, 4096, 4096, 0, 0, C.byref(n)) == P.OK and n.value == 0
    assert L.comp_ams_linear_q8_work_bytes(4, 131_072, 4096, 1, 1, C.byref(n)) == P.EINVAL and L.comp_ams_linear_q8_work_bytes(4, 5, 6, 0, 0, None) == P.EINVAL
    assert L.comp_ams_linear_weight_grad_work_bytes(4096, 768, 768, 8, 1, 1, 1, C.byref(n)) == P.OK
    assert L.comp_ams_linear_weight_grad_work_bytes(4096, 768, 768, 7, 1, 1, 1, C.byref(n)) == P.EINVAL
    assert L.comp_ams_linear_weight_grad_work_bytes(4096, 768, 768, 8, 1, 7, 1, C.byref(n)) == P.EINVAL
    assert L.comp_ams_linear_weight_grad_work_bytes(4096, 768, 768, 8, 1, 1, 0, None) == P.EINVAL


def test_the_python_entry_points_refuse():
    x, f = torch.zeros(4, 8), torch.zeros(8)
    q, s = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)
    w, ws = torch.zeros(6, 8, dtype=torch.int8), torch.zeros(6)
    dw, dy = torch.zeros(2, 6, 8), torch.zeros(4, 6)
    calls = [
        lambda: P.quantize_rows(x), lambda: P.quantize_rows(x.double()), lambda: P.quantize_rows(x.t()), lambda: P.quantize_rows(q),      # the first: not on the GPU
        lambda: P.restore_rows(x, s), lambda: P.restore_rows(q, s[:3]), lambda: P.restore_rows(q, s.double()), lambda: P.restore_rows(q.t(), f),
        lambda: P.rms_norm(x, f), lambda: P.rms_norm(x, f[:7]), lambda: P.rms_norm(x, f.double()), lambda: P.rms_norm(x, f, x[:3]), lambda: P.rms_norm(x, f, x.half()),
        lambda: P.rms_norm(q, f), lambda: P.rms_norm_q8(x.double(), f), lambda: P.rms_norm_q8(x, f, x[:, :4]),
        lambda: P.rms_norm_backward(x, x[:3], s, f, x[:2]), lambda: P.rms_norm_backward(x, q, s, f, x[:2]), lambda: P.rms_norm_backward(x, x, s, f, x[:2], scale=s),
        lambda: P.rms_norm_backward(x, q, s, f, x[:2], scale=s[:2]), lambda: P.rms_norm_backward(x, x, s[:3], f, x[:2]), lambda: P.rms_norm_backward(x, x, s, f, x[:2, :7]),
        lambda: P.rms_norm_backward(x, x, s, f, x[:2], x[:2]), lambda: P.rms_norm_backward(x, x.half(), s, f, x[:2]),
        lambda: P.linear_q8(q, s, w, ws), lambda: P.linear_q8(x, s, w, ws), lambda: P.linear_q8(q, s, w.float(), ws), lambda: P.linear_q8(q, s, w[:, :7], ws),
        lambda: P.linear_q8(q, s[:3], w, ws), lambda: P.linear_q8(q, s, w, ws[:5]), lambda: P.linear_q8(q, s, w, ws, ws[:5]), lambda: P.linear_q8(q, s, w, ws, out=dy.t()),
        lambda: P.linear_q8(q, s, w, ws, dtype=torch.float64), lambda: P.linear_q8(q, s, w, ws, dtype=torch.float16, out=dy), lambda: P.linear_q8(q, s, w.t(), ws),
        lambda: P.linear_weight_grad(dy, q, s, dw), lambda: P.linear_weight_grad(dy[:3], q, s, dw), lambda: P.linear_weight_grad(dy, x, s, dw),
        lambda: P.linear_weight_grad(dy, q, s[:2], dw), lambda: P.linear_weight_grad(dy, q, s, dw[:, :5]), lambda: P.linear_weight_grad(dy, q, s, dw[0]),
        lambda: P.linear_weight_grad(dy, q, s, torch.zeros(2, 6, 16)[:, :, ::2]), lambda: P.linear_weight_grad(dy, q, s, torch.zeros(2, 7, 8)[:, :6].transpose(1, 2).contiguous()),
        lambda: P.linear_weight_grad(dy, q, s, dw, torch.zeros(2, 5)), lambda: P.linear_weight_grad(dy, q, s, dw, torch.zeros(2, 6)),
        lambda: P.linear_weight_grad(dy, q, s, dw, torch.zeros(2, 6).half()), lambda: P.linear_weight_grad(dy.double(), q, s, dw),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} went through")
