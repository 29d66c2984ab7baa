"""The operators of include/comp_ams_rows8.h through the C functions: what the header allows and the Python entry points never pass."""
import ctypes as C
import zlib

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P
import rows8_util as Q

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CODE = {F32: 0, BF16: 1, F16: 2}


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def call(name, *args):
    stream = torch.cuda.current_stream().cuda_stream
    rc = getattr(P.lib(), "comp_ams_" + name)(*(a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args), stream)
    assert rc == P.OK, P.lib().comp_ams_operators_last_error().decode()


def work_memory(name, *args):
    need = C.c_uint64(0)
    assert getattr(P.lib(), f"comp_ams_{name}_work_bytes")(*args, C.byref(need)) == P.OK
    return torch.empty(max(need.value, 16), dtype=torch.uint8, device="cuda"), need.value


@pytest.mark.parametrize("binary", [1, 0])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("cols,outs", [(40, 64), (300, 256), (24, 600), (9, 17)])
def test_linear_weight_grad_of_one_row_with_any_stride(cols, outs, dtype, binary):
    """One row has no next one: its stride, of dy and of q, says nothing."""
    print(f"[case] one row {cols}->{outs} {dtype} {binary}", flush=True)
    g = gen("one row", cols, outs)
    q, scale = Q.quantized(torch.randn(1, cols, generator=g), True)
    dy = (torch.randn(1, outs, generator=g) * 0.1).to(dtype)
    dw, db, s_dw, s_db = Q.weight_grad(dy, q, scale, 1, binary)
    work, size = work_memory("linear_weight_grad", 1, cols, outs, 1, binary, CODE[dtype], 1 if outs % 8 == 0 else 0)
    qc, sc, dyc = q.cuda(), scale.cuda(), dy.cuda()
    for dy_stride, q_stride in ((outs, cols), (0, 0), (8, 1), (outs - 1, cols), (outs + 3, 1 << 40), (1 << 31, cols), (3 << 29, cols), (1 << 59, 1 << 59)):
        for in_first in (0, 1):
            w, b = torch.full((outs * cols,), 7.0, device="cuda"), torch.full((outs,), 7.0, device="cuda")
            call("linear_weight_grad", w, b, dyc, qc, sc, 1, cols, outs, dy_stride, q_stride, 1, 0, in_first, binary, CODE[dtype], 0, work, size)
            got = w.view(cols, outs).t() if in_first else w.view(outs, cols)
            R.close(got, dw[0], s_dw[0], f"dweight, stride {dy_stride}")
            R.close(b, db[0], s_db[0], f"dbias, stride {dy_stride}")


@pytest.mark.parametrize("cols,outs", [(12, 8), (33, 24), (300, 200)])
def test_linear_weight_grad_of_aligned_rows_that_nobody_promised(cols, outs):
    """bfloat16 and scales of any value: of aligned dy the input may take the planes, for which there has to be room."""
    print(f"[case] no promise {cols}->{outs}", flush=True)
    g = gen("no promise", cols, outs)
    rows, n = 128, 2
    q, scale = Q.quantized(torch.randn(rows, cols, generator=g), False)
    dy = (torch.randn(rows, outs, generator=g) * 0.1).to(BF16)
    dw, _, s_dw, _ = Q.weight_grad(dy, q, scale, n, False)
    work, size = work_memory("linear_weight_grad", rows, cols, outs, n, 0, 1, 0)
    w = torch.zeros(n, outs, cols, device="cuda")
    call("linear_weight_grad", w, None, dy.cuda(), q.cuda(), scale.cuda(), rows, cols, outs, outs, cols, n, outs * cols, 0, 0, 1, 0, work, size)
    R.close(w, dw, s_dw, "dweight")
    far = torch.zeros(rows, 1 << 22, dtype=BF16, device="cuda")[:, :outs]                  # aligned rows further apart than the binding promises
    far.copy_(dy)
    again = torch.zeros_like(w)
    P.linear_weight_grad(far, q.cuda(), scale.cuda(), again)
    assert R.same_bits(again, w)


# rows that a team of lanes holds, of one wavefront and of several, with ends inside a lane's numbers, and rows of any length
IN_PLACE = [(40, 100, F32), (33, 1000, BF16), (20, 2047, F32), (9, 8190, F16), (7, 9001, BF16), (5, 17_001, BF16), (3, 70_001, F32), (6, 5, BF16), (4500, 2049, F32)]


@pytest.mark.parametrize("rows,cols,dtype", IN_PLACE, ids=str)
def test_rms_norm_whose_sum_or_result_takes_the_place_of_an_input(rows, cols, dtype):
    print(f"[case] in place {rows}x{cols} {dtype}", flush=True)
    g = gen("in place", rows, cols)
    x, res, gain = torch.randn(rows, cols, generator=g).to(dtype).cuda(), torch.randn(rows, cols, generator=g).to(dtype).cuda(), torch.randn(cols, generator=g).cuda()
    want_y, want_h, want_r = P.rms_norm(x, gain, res)
    want_q, want_s, _, _ = P.rms_norm_q8(x, gain, res)
    alone, _, alone_r = P.rms_norm(x, gain)
    rstd, scale = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")

    def norm(y, h, a, b):
        call("rms_norm", y, h, rstd, a, b, gain, rows, cols, cols, cols, cols, cols, 1e-5, CODE[dtype])

    for which in (0, 1):                                                # h in the place of x, or of the residual; y in the other one's, or in its own
        for both in (False, True):
            ins = [x.clone(), res.clone()]
            y = ins[1 - which] if both else torch.zeros_like(x)
            norm(y, ins[which], *ins)
            assert R.same_bits(y, want_y) and R.same_bits(ins[which], want_h) and R.same_bits(rstd, want_r)
        ins = [x.clone(), res.clone()]                                  # y in an input's place, h not stored, or elsewhere
        norm(ins[which], None, *ins)
        assert R.same_bits(ins[which], want_y)
        ins, h = [x.clone(), res.clone()], torch.zeros_like(x)
        norm(ins[which], h, *ins)
        assert R.same_bits(ins[which], want_y) and R.same_bits(h, want_h)
        ins, q = [x.clone(), res.clone()], torch.zeros(rows, cols, dtype=torch.int8, device="cuda")
        call("rms_norm_q8", q, scale, ins[which], rstd, *ins, gain, rows, cols, cols, cols, cols, cols, 1e-5, 0, CODE[dtype])
        assert torch.equal(q, want_q) and R.same_bits(scale, want_s) and R.same_bits(ins[which], want_h) and R.same_bits(rstd, want_r)
    again = x.clone()                                                   # no residual: y in the place of x
    norm(again, None, again, None)
    assert R.same_bits(again, alone) and R.same_bits(rstd, alone_r)
    h = torch.zeros_like(x)
    norm(h.clone(), h, x, None)
    assert R.same_bits(h, x)
