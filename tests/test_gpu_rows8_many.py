"""The operators on rows in 8 bits where workgroups go on to further rows, and where arrays are large enough to pass the caches by: beyond 16 MiB (the
norm's h), 48 MiB (its inputs), 80 MiB (results) and 256 MiB (rows to 8 bits).  The 64-bit forms are computed on the GPU."""
import zlib

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P
import rows8_util as Q

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def generator(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def randn(g, *shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda") * std


def near(got, want, slack, what):
    """R.close for finite values, without leaving the GPU."""
    off = (got.double() - want).abs() - (2 * R.U[got.dtype] * want.abs() + R.TINY[got.dtype] + slack)
    assert not torch.isnan(off).any() and float(off.max()) <= 0, f"{what}: off by {float(off.max())} too much in {int((off > 0).sum())} of {off.numel()}"


# teams of 16, 64, 256, 512 and 1024 lanes, more than the 4096 workgroups of a launch have at a time; the last two go past the caches
MANY = [(70_000, 100, F32), (17_001, 1000, BF16), (5000, 2047, F32), (4301, 8000, F16), (4800, 9001, BF16), (4200, 17_001, BF16), (4100, 9005, F32)]


@pytest.mark.parametrize("rows,cols,dtype", MANY, ids=str)
def test_norm_of_many_rows(rows, cols, dtype):
    print(f"[case] rms {rows}x{cols} {dtype}", flush=True)
    g = generator("many", rows, cols)
    x, res, gain = (randn(g, rows, cols, std=1.5) + randn(g, rows, 1)).to(dtype), randn(g, rows, cols, std=2.0).to(dtype), randn(g, cols)
    for r in (res, None):
        want, h, rstd, slack, s_rstd = Q.rms(x, r, gain, 1e-5)
        y, got_h, got_r = P.rms_norm(x, gain, r)
        assert R.same_bits(got_h, h)
        near(y, want, slack, "y")
        near(got_r, rstd, s_rstd, "rstd")
        q, scale, h8, r8 = P.rms_norm_q8(x, gain, r, binary=r is None)
        assert R.same_bits(h8, h) and R.same_bits(r8, got_r)
        top, loose = want.abs().amax(-1), slack.amax(-1) / 127 + 4 * Q.E32 * want.abs().amax(-1)
        if r is None:
            assert (torch.frexp(scale)[0] == 0.5).all() and (scale.double() >= top / 127 - loose).all() and (scale.double() / 2 < top / 127 + loose).all()
        else:
            assert ((scale.double() - top / 127).abs() <= loose).all()
        assert ((q.double() * scale.double()[:, None] - want).abs() <= scale.double()[:, None] * (0.5 + 512 * Q.E32) + slack + loose[:, None]).all()
        del want, slack


@pytest.mark.parametrize("rows,cols,dtype", MANY, ids=str)
def test_norm_backward_of_many_rows(rows, cols, dtype):
    print(f"[case] rms backward {rows}x{cols} {dtype}", flush=True)
    g = generator("many backward", rows, cols)
    n = 2 if rows % 2 == 0 else 1
    h, gain = randn(g, rows, cols, std=1.5).to(dtype), randn(g, cols)
    dy, past = randn(g, rows, cols, std=0.3).to(dtype), randn(g, rows, cols, std=0.3).to(dtype)
    rstd = (1 / ((h.double() ** 2).mean(-1) + 1e-5).sqrt()).float()
    q, scale = P.quantize_rows(h)
    for kept, s in ((h, None), (q, scale)):
        stood = kept if s is None else kept.float() * s[:, None]
        dx, dgain, s_dx, s_gain = Q.rms_backward(dy, stood, rstd, gain, past, n)
        got_gain = torch.zeros(n, cols, device="cuda")
        near(P.rms_norm_backward(dy, kept, rstd, gain, got_gain, past, s), dx, s_dx, "dx")
        near(got_gain, dgain, s_gain, "dgain")
        del dx, s_dx


@pytest.mark.parametrize("binary", [False, True])
@pytest.mark.parametrize("rows,cols,dtype", [(5000, 27_003, BF16), (8500, 16_001, F16), (8195, 8200, F32), (135_001, 1001, BF16), (1_500_001, 45, F32)], ids=str)
def test_rows_past_the_caches(rows, cols, dtype, binary):
    print(f"[case] rows8 {rows}x{cols} {dtype} {binary}", flush=True)
    g = generator("past", rows, cols)
    x = (randn(g, rows, cols) * torch.exp(randn(g, rows, 1))).to(dtype)
    assert x.numel() * x.element_size() > 256 << 20
    q, scale = P.quantize_rows(x, binary=binary)
    some = torch.cat([torch.arange(64), torch.randint(0, rows, (64,)), torch.arange(rows - 64, rows)]).cuda()
    want_q, want_s = Q.quantized(x[some], binary)
    assert torch.equal(q[some].cpu(), want_q) and torch.equal(scale[some].cpu(), want_s)
    top = x.float().abs().amax(-1).double() / 127                       # all of them: the scale, and half a step
    assert ((scale.double() >= top * (1 - Q.E32)) & (scale.double() <= (2 if binary else 1) * top * (1 + Q.E32))).all()
    assert ((q.float() * scale[:, None] - x.float()).abs() <= scale[:, None] * 0.50002).all()
    assert R.same_bits(P.restore_rows(q, scale, dtype), (q.float() * scale[:, None]).to(dtype))


@pytest.mark.parametrize("rows,cols,outs,dtype", [(5000, 64, 8512, BF16), (5003, 77, 4512, F32), (1700, 272, 25_024, F16)], ids=str)
def test_product_past_the_caches(rows, cols, outs, dtype):
    print(f"[case] product {rows}x{cols}x{outs} {dtype}", flush=True)
    g = generator("past product", rows, cols, outs)
    whole = lambda *shape: torch.randint(-128, 128, shape, generator=g, dtype=torch.int16, device="cuda").to(torch.int8)
    q, w = whole(rows, cols), whole(outs, cols)
    s, ws = torch.exp(randn(g, rows) * 0.5) * 0.002, torch.exp(randn(g, outs) * 0.5) * 0.2
    want = (q.double() @ w.double().t().contiguous()) * s.double()[:, None] * ws.double()
    y = P.linear_q8(q, s, w, ws, dtype=dtype)
    assert y.numel() * y.element_size() > 80 << 20 and y.data_ptr() % 128 == 0 and y.stride(0) * y.element_size() % 128 == 0
    near(y, want, 4 * Q.E32 * want.abs(), "y")
    odd = torch.full((rows, outs + 1), 7.0, dtype=dtype, device="cuda")  # through the caches: rows that share lines
    P.linear_q8(q, s, w, ws, out=odd[:, :outs])
    assert R.same_bits(odd[:, :outs], y) and (odd[:, outs] == 7).all()


@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("n,per,cols,outs", [(1, 100, 4800, 9001), (2, 130, 4801, 4544), (4, 33, 3264, 3300)], ids=str)
def test_weight_gradients_past_the_caches(n, per, cols, outs, grad):
    print(f"[case] weights {n}x{per} {cols}->{outs} {grad}", flush=True)
    g = generator("past weights", n, per, cols, outs)
    rows = n * per
    q, scale = P.quantize_rows(randn(g, rows, cols), binary=True)
    dy = randn(g, rows, outs, std=0.1).to(BF16)
    dw, db, s_dw, s_db = Q.weight_grad(dy, q, scale, n, True)
    size = outs * cols
    for turned in (False, True):
        place = torch.full((n, (size + outs + 127) // 64 * 64), 7.0, dtype=grad, device="cuda")          # the workers' rows begin at whole lines
        w, b = place[:, :size], place[:, size:size + outs]
        w = w.unflatten(1, (cols, outs)).transpose(1, 2) if turned else w.unflatten(1, (outs, cols))
        assert n * size * place.element_size() > 80 << 20
        P.linear_weight_grad(dy, q, scale, w, b, binary=True)
        near(w, dw, s_dw, f"dweight {turned}")
        near(b, db, s_db, "dbias")
        assert (place[:, size + outs:] == 7).all()
