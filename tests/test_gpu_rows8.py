"""The operators of include/comp_ams_rows8.h against plain 64-bit forms, through the Python entry points: types, sizes from one element
to long rows, strides, ends inside a vector or a tile, extremes, workers, and what must not be touched."""
import zlib

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P
import rows8_util as Q

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DTYPES = [F32, BF16, F16]
SIZES = [(1, 1), (3, 2), (5, 7), (4, 16), (9, 33), (2, 64), (7, 130), (3, 255), (3, 256), (6, 257), (5, 511), (5, 512), (4, 768), (3, 1023), (3, 1025),
         (2, 2047), (2, 2049), (2, 4099), (2, 8192), (2, 8193), (3, 12_001), (2, 16_001), (1, 16_385), (2, 24_001), (1, 30_003), (1, 33_001), (2, 70_001), (3000, 24), (2500, 1000)]


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def randn(g, *shape, std=1.0):
    return torch.randn(shape, generator=g) * std


def strided(t, pad=0, lead=0, fill=9):
    """t's values on the GPU inside a larger array: rows `pad` elements further apart, `lead` elements in front."""
    rows, cols = t.shape
    buf = torch.full((lead + rows * (cols + pad) + 40,), fill, dtype=t.dtype, device="cuda")
    view = buf[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view, buf


def around(buf, rows, cols, pad, lead, fill=9):
    keep = torch.ones(buf.numel(), dtype=torch.bool)
    keep[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = False
    assert (buf.cpu()[keep] == fill).all(), "wrote outside the rows"


def same(a, b):
    """Equal, a NaN to a NaN."""
    a, b = a.cpu(), b.cpu()
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.where(torch.isnan(a), 0, a), torch.where(torch.isnan(b), 0, b))


# --- rows to 8 bits and back ----------------------------------------------------------------------------------------

def rows_of_all_kinds(g, rows, cols, dtype):
    x = randn(g, rows, cols) * torch.exp(3 * randn(g, rows, 1))
    if rows > 2:
        x[1] = 0
    return x.to(dtype)


@pytest.mark.parametrize("binary", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantize_and_restore(rows, cols, dtype, binary):
    print(f"[case] rows {rows}x{cols} {dtype} {binary}", flush=True)
    g = gen("rows8", rows, cols)
    x = rows_of_all_kinds(g, rows, cols, dtype)
    want_q, want_s = Q.quantized(x, binary)
    for view in (x.cuda(), strided(x, pad=3, lead=1, fill=float("nan"))[0]):
        q, s = P.quantize_rows(view, binary=binary)
        assert torch.equal(q.cpu(), want_q) and same(s, want_s)
    qv, _ = strided(want_q, pad=5, lead=3)
    for to in DTYPES:
        out, buf = strided(torch.zeros(rows, cols, dtype=to), pad=1, lead=3)
        got = P.restore_rows(qv, want_s.cuda(), out=out)
        assert same(got, (want_q.float() * want_s[:, None]).to(to))
        around(buf, rows, cols, 1, 3)
        assert same(P.restore_rows(q, s, to), out)
    if binary:
        exact = want_q.double() * want_s.double()[:, None]
        assert same(P.restore_rows(q, s, F32).double(), exact) and same(P.restore_rows(q, s, BF16).double(), exact)


@pytest.mark.parametrize("binary", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_extremes(dtype, binary):
    big = torch.finfo(dtype).max
    small = torch.finfo(dtype).smallest_normal
    rows = [[0.0, -0.0] * 8, [big, -big] + [1.0] * 14, [big * 0.99] + [-big / 3] * 15, [small] * 15 + [-small], [small * 2 ** -6] * 16,
            [1.0, 0.5, -1.5, 2.5] * 4, [127.0, 0.5, 1.5, 2.5] + [-0.5] * 12]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype)
    q, s = P.quantize_rows(x.cuda(), binary=binary)
    want = Q.quantized(x, binary)
    assert torch.equal(q.cpu(), want[0]) and torch.equal(s.cpu(), want[1])
    back = P.restore_rows(q, s, dtype).cpu()
    assert torch.isfinite(back).all()
    # within a rounding to the type of half a step of the row's scale, a whole one where 127 steps would leave the type
    assert ((back.double() - x.double()).abs() <= s.cpu().double()[:, None] * (1 + 2.0 ** -7) + R.U[dtype] * 2 * x.double().abs()).all()
    for bad in (float("inf"), -float("inf"), float("nan")):
        y = torch.ones(3, 40, dtype=dtype)
        y[1, 37] = bad
        q, s = P.quantize_rows(y.cuda(), binary=binary)
        assert torch.isnan(s[1]) and (q[1] == 0).all() and torch.isfinite(s[[0, 2]]).all()
        back = P.restore_rows(q, s, dtype).cpu()
        assert torch.isnan(back[1]).all() and torch.isfinite(back[[0, 2]]).all()


def test_rows8_shapes():
    for shape in ((0, 5), (3, 0), (0, 0), (2, 0, 4), (7,), (2, 3, 9)):
        x = randn(gen(shape), *shape).cuda()
        q, s = P.quantize_rows(x)
        assert q.shape == x.shape and s.shape == x.shape[:-1]
        assert P.restore_rows(q, s).shape == x.shape
        want = Q.quantized(x, False)
        assert torch.equal(q.cpu(), want[0]) and torch.equal(s.cpu(), want[1])


# --- the norm ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rms_norm(rows, cols, dtype):
    print(f"[case] rms {rows}x{cols} {dtype}", flush=True)
    g = gen("rms", rows, cols)
    x = (randn(g, rows, cols, std=1.5) + randn(g, rows, 1)).to(dtype)
    res, gain = randn(g, rows, cols, std=2.0).to(dtype), randn(g, cols)
    xv, rv = strided(x, 3, 1, float("nan"))[0], strided(res, 2, 5, float("nan"))[0]
    for r, view in ((res, rv), (None, None)):
        y, h, rstd, slack, s_rstd = Q.rms(x, r, gain, 1e-5)
        out, buf = strided(torch.zeros_like(x), 5, 3)
        got = P.rms_norm(xv, gain.cuda(), view, out=out)
        assert got[0] is out and torch.equal(got[1].cpu(), h) and (r is not None or got[1] is xv)
        R.close(got[0], y, slack, "y")
        R.close(got[2], rstd, s_rstd, "rstd")
        around(buf, rows, cols, 5, 3)
        dense = P.rms_norm(x.cuda(), gain.cuda(), None if r is None else r.cuda())
        assert R.same_bits(dense[0], out) and R.same_bits(dense[2], got[2])
        for binary in (False, True):
            q, scale, h8, rstd8 = P.rms_norm_q8(xv, gain.cuda(), view, binary=binary)
            assert torch.equal(h8.cpu(), h) and R.same_bits(rstd8, got[2])
            Q.check_q8(q, scale, y, slack, binary)
    into, like = res.cuda(), P.rms_norm(x.cuda(), gain.cuda(), res.cuda())
    got = P.rms_norm(x.cuda(), gain.cuda(), into, out=into)                  # y in the residual's place
    assert R.same_bits(got[0], like[0]) and got[0] is into


def test_rms_norm_of_nothing_but_zeros():
    for dtype in DTYPES:
        x = torch.zeros(3, 100, dtype=dtype, device="cuda")
        y, h, rstd = P.rms_norm(x, torch.ones(100, device="cuda"), eps=1e-5)
        assert (y == 0).all() and torch.allclose(rstd.cpu(), torch.full((3,), 1e-5 ** -0.5))
        q, scale, _, _ = P.rms_norm_q8(x, torch.ones(100, device="cuda"))
        assert (q == 0).all() and (scale == Q.LEAST).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,per,cols", [(1, 1, 1), (3, 2, 7), (2, 5, 33), (1, 40, 64), (4, 33, 130), (2, 3, 256), (5, 7, 511), (8, 20, 768), (2, 2, 1025), (3, 9, 2047),
                                        (2, 3, 4099), (1, 4, 8193), (2, 1, 33_001), (20, 100, 96), (1, 3000, 48), (2, 3, 12_001), (1, 5, 16_003), (3, 9, 1000), (1, 33, 100), (2, 2, 9001),
                                        (1, 700, 1030)])
def test_rms_norm_backward(n, per, cols, dtype):
    print(f"[case] rms backward {n}x{per}x{cols} {dtype}", flush=True)
    g = gen("rmsb", n, per, cols)
    rows = n * per
    h = randn(g, rows, cols, std=1.5).to(dtype)
    dy, past, gain = randn(g, rows, cols, std=0.3).to(dtype), randn(g, rows, cols, std=0.3).to(dtype), randn(g, cols)
    rstd = (1 / ((h.double() ** 2).mean(-1) + 1e-5).sqrt()).float()
    q, scale = Q.quantized(h, False)
    for kept8 in (False, True):
        stood = q.float() * scale[:, None] if kept8 else h
        hv = strided(q if kept8 else h, 7, 1, 9)[0]
        for r in (past, None):
            dx, dgain, s_dx, s_gain = Q.rms_backward(dy, stood, rstd, gain, r, n)
            for grad in (F32, BF16, F16):
                buf = torch.full((n, 3 + cols + 4), 7.0, dtype=grad, device="cuda")
                out, obuf = strided(torch.zeros_like(dy), 1, 3)
                got = P.rms_norm_backward(strided(dy, 2, 1, float("nan"))[0], hv, rstd.cuda(), gain.cuda(), buf[:, 3:3 + cols],
                                          None if r is None else strided(r, 4, 3, float("nan"))[0], scale.cuda() if kept8 else None, out=out)
                R.close(got, dx, s_dx, "dx")
                R.close(buf[:, 3:3 + cols], dgain, s_gain, "dgain")
                assert (buf[:, :3] == 7).all() and (buf[:, 3 + cols:] == 7).all()
                around(obuf, rows, cols, 1, 3)
    grads = torch.zeros(n, cols, device="cuda")
    want = P.rms_norm_backward(dy.cuda(), h.cuda(), rstd.cuda(), gain.cuda(), grads, past.cuda())
    for which in range(3):                                                     # dx in the place of dy, h or dresidual
        a = [dy.cuda(), h.cuda(), past.cuda()]
        again = torch.zeros_like(grads)
        got = P.rms_norm_backward(a[0], a[1], rstd.cuda(), gain.cuda(), again, a[2], out=a[which])
        assert R.same_bits(got, want) and R.same_bits(again, grads)


def test_rms_norm_gradient_against_differences():
    g = gen("diff")
    x, gain, up = randn(g, 6, 37).double(), randn(g, 37).double(), randn(g, 6, 37).double()
    f = lambda xx, gg: float((xx / ((xx ** 2).mean(-1, keepdim=True) + 1e-5).sqrt() * gg * up).sum())
    y, h, rstd = P.rms_norm(x.float().cuda(), gain.float().cuda())
    dgain = torch.zeros(1, 37, device="cuda")
    dx = P.rms_norm_backward(up.float().cuda(), h, rstd, gain.float().cuda(), dgain)
    step = 1e-5
    for r, c in ((0, 0), (2, 17), (5, 36)):
        e = torch.zeros_like(x)
        e[r, c] = step
        assert abs((f(x + e, gain) - f(x - e, gain)) / (2 * step) - float(dx[r, c])) < 1e-4
    for c in (0, 20, 36):
        e = torch.zeros_like(gain)
        e[c] = step
        assert abs((f(x, gain + e) - f(x, gain - e)) / (2 * step) - float(dgain[0, c])) < 1e-4


# --- the product ------------------------------------------------------------------------------------------------------

def whole(g, *shape):
    return torch.randint(-128, 128, shape, generator=g, dtype=torch.int16).to(torch.int8)


PRODUCTS = [(1, 1, 1), (1, 64, 16), (3, 7, 5), (16, 128, 48), (17, 130, 33), (5, 4096, 100), (33, 1000, 70), (64, 2048, 257), (48, 1024, 16), (65, 16, 3),
            (65, 128, 128), (100, 1, 130), (129, 15, 127), (200, 272, 640), (130, 1111, 500), (300, 4096, 300), (1000, 96, 1000), (257, 144, 255), (70, 3000, 65)]


@pytest.mark.parametrize("rows,cols,outs", PRODUCTS)
def test_linear_q8(rows, cols, outs):
    print(f"[case] product {rows}x{cols}x{outs}", flush=True)
    g = gen("product", rows, cols, outs)
    q, w = whole(g, rows, cols), whole(g, outs, cols)
    s, ws, bias = torch.exp(randn(g, rows)) * 0.01, torch.exp(randn(g, outs)) * 0.02, randn(g, outs)
    for b in (None, bias):
        want, slack = Q.linear(q, s, w, ws, b)
        bc = None if b is None else b.cuda()
        for dtype in DTYPES:
            if dtype == F16:
                want, slack = want * 2.0 ** -8, slack * 2.0 ** -8                 # within its range
            sc = (s * 2.0 ** -8 if dtype == F16 else s).cuda()
            if dtype == F16 and b is not None:
                bc = (b * 2.0 ** -8).cuda()
            first = None
            # dense; 16-byte strides; odd strides and addresses
            for pad, lead in ((0, 0), (48, 32), (5, 3)):
                qv, wv = strided(q, pad, lead)[0], strided(w, pad, lead)[0]
                out, buf = strided(torch.zeros(rows, outs, dtype=dtype), 3, 1)
                got = P.linear_q8(qv, sc, wv, ws.cuda(), bc, out=out)
                assert got is out
                R.close(got, want, slack, f"{dtype} {pad}")
                around(buf, rows, outs, 3, 1)
                first = got.clone() if first is None else first
                assert R.same_bits(got, first)                                    # exact sums: every path gives the same bits
            assert R.same_bits(P.linear_q8(q.cuda(), sc, w.cuda(), ws.cuda(), bc, dtype=dtype), first)


# the tiles of 256 x 256, 256 x 128, 128 x 128 and 64 x 128, and k in pieces, each over sizes that end inside a tile
@pytest.mark.parametrize("rows,cols,outs", [(3600, 80, 3700), (3585, 77, 3599), (4000, 400, 3400), (2000, 208, 4100), (2040, 131, 4001), (1000, 200, 4090), (500, 333, 4000),
                                            (100, 8200, 1000), (70, 16_400, 130), (40, 20_000, 65)])
def test_linear_q8_large_tiles(rows, cols, outs):
    print(f"[case] product {rows}x{cols}x{outs}", flush=True)
    g = gen("large", rows, cols, outs)
    q, w = whole(g, rows, cols).cuda(), whole(g, outs, cols).cuda()
    s, ws = (torch.exp(randn(g, rows)) * 0.01).cuda(), (torch.exp(randn(g, outs)) * 0.02).cuda()
    y = P.linear_q8(q, s, w, ws, dtype=F32)
    acc = q.double() @ w.double().t().contiguous()
    want = acc * s.double()[:, None] * ws.double()
    assert ((y.double() - want).abs() <= 6 * Q.E32 * want.abs()).all()


def test_linear_q8_sums_stay_exact():
    cols = 131_071
    for rows in (2, 70):
        q = torch.full((rows, cols), -128, dtype=torch.int8, device="cuda")
        w = torch.full((5, cols), -128, dtype=torch.int8, device="cuda")
        w[1] = 127
        w[2, 7:] = 0
        one = torch.ones(max(rows, 5), device="cuda")
        y = P.linear_q8(q, one[:rows], w, one[:5], dtype=F32)
        want = torch.tensor([16384.0 * cols, -16256.0 * cols, 16384.0 * 7, 16384.0 * cols, 16384.0 * cols], dtype=torch.float64).float()
        assert torch.equal(y.cpu(), want.expand(rows, 5))
    with pytest.raises(P.CompAmsError, match="cols"):
        P.linear_q8(torch.zeros(1, 131_072, dtype=torch.int8, device="cuda"), one[:1], torch.zeros(1, 131_072, dtype=torch.int8, device="cuda"), one[:1])


def test_linear_q8_of_nothing():
    one = torch.ones(9, device="cuda")
    z = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda")
    assert P.linear_q8(z(0, 8), one[:0], z(5, 8), one[:5]).shape == (0, 5)
    assert P.linear_q8(z(3, 8), one[:3], z(0, 8), one[:0]).shape == (3, 0)
    for rows in (3, 70):
        many = torch.ones(rows, device="cuda")
        assert torch.equal(P.linear_q8(z(rows, 0), many, z(5, 0), one[:5], bias=one[:5] * 3, dtype=F32), torch.full((rows, 5), 3.0, device="cuda"))
    assert P.linear_q8(z(2, 3, 8), torch.ones(2, 3, device="cuda"), z(5, 8), one[:5]).shape == (2, 3, 5)


def test_linear_q8_nan_scales_stay_with_their_rows_and_channels():
    g = gen("nan")
    q, w = whole(g, 70, 100).cuda(), whole(g, 40, 100).cuda()
    s, ws = torch.ones(70, device="cuda"), torch.ones(40, device="cuda")
    s[3], ws[7] = float("nan"), float("inf")
    bad = torch.isfinite(P.linear_q8(q, s, w, ws, dtype=F32)).cpu()
    want = torch.ones(70, 40, dtype=torch.bool)
    want[3], want[:, 7] = False, False
    assert torch.equal(bad, want)


# --- weight gradients ---------------------------------------------------------------------------------------------------

WEIGHTS = [(1, 1, 1, 1), (2, 3, 5, 7), (1, 32, 16, 16), (3, 33, 17, 130), (2, 64, 128, 128), (1, 100, 129, 127), (4, 31, 300, 20), (1, 1000, 64, 200), (2, 700, 257, 255),
           (20, 10, 40, 33), (1, 4000, 130, 15)]


@pytest.mark.parametrize("binary", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,per,cols,outs", WEIGHTS)
def test_linear_weight_grad(n, per, cols, outs, dtype, binary):
    print(f"[case] weights {n}x{per} {cols}->{outs} {dtype} {binary}", flush=True)
    g = gen("weights", n, per, cols, outs)
    rows = n * per
    q, scale = Q.quantized(randn(g, rows, cols) * torch.exp(randn(g, rows, 1)), binary)
    dy = randn(g, rows, outs, std=0.1).to(dtype)
    dw, db, s_dw, s_db = Q.weight_grad(dy, q, scale, n, binary)
    d = 3 + outs * cols + outs + 2
    for pad, lead in ((0, 0), (5, 3)):
        qv, dyv = strided(q, pad, lead)[0], strided(dy, pad, lead, float("nan"))[0]
        for grad in DTYPES:
            for turned in (False, True):
                buf = torch.full((n, d), 7.0, dtype=grad, device="cuda")
                place = buf[:, 3:3 + outs * cols]
                w = place.unflatten(1, (cols, outs)).transpose(1, 2) if turned else place.unflatten(1, (outs, cols))
                b = buf[:, 3 + outs * cols:-2]
                P.linear_weight_grad(dyv, qv, scale.cuda(), w, b, binary=binary)
                R.close(w, dw, s_dw, f"dweight {grad} {turned}")
                R.close(b, db, s_db, "dbias")
                assert (buf[:, :3] == 7).all() and (buf[:, -2:] == 7).all()
    first = torch.zeros(n, outs, cols, device="cuda")
    P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), first, binary=binary)
    again = torch.zeros_like(first)
    P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), again, binary=binary)
    assert R.same_bits(first, again)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,per,cols,outs", [(8, 64, 1300, 1290), (1, 96, 3600, 3700), (4, 70, 2047, 1801), (1, 500, 2040, 2000), (1, 9000, 1000, 1030),
                                                   (2, 5000, 300, 200), (3, 2000, 70, 520)])
def test_linear_weight_grad_large_tiles(n, per, cols, outs, dtype):
    print(f"[case] weights {n}x{per} {cols}->{outs} {dtype}", flush=True)
    g = gen("weights large", n, per, cols, outs)
    q, scale = Q.quantized(randn(g, n * per, cols), True)
    dy = randn(g, n * per, outs, std=0.1).to(dtype)
    q, scale, dy = q.cuda(), scale.cuda(), dy.cuda()
    dw, _, s_dw, _ = Q.weight_grad(dy, q, scale, n, True)
    for turned in (False, True):
        got = torch.zeros(n, cols, outs, device="cuda").transpose(1, 2) if turned else torch.zeros(n, outs, cols, device="cuda")
        P.linear_weight_grad(dy, q, scale, got, binary=True)
        assert ((got.double() - dw).abs() <= s_dw + 2 * Q.E32 * dw.abs()).all()


def test_linear_weight_grad_of_nothing():
    z = lambda *s, t=F32: torch.zeros(s, dtype=t, device="cuda")
    dw, db = torch.full((2, 4, 3), 5.0, device="cuda"), torch.full((2, 4), 5.0, device="cuda")
    grads = torch.full((2, 16), 5.0, device="cuda")
    P.linear_weight_grad(z(0, 4), z(0, 3, t=torch.int8), z(0), grads[:, :12].unflatten(1, (4, 3)), grads[:, 12:])
    assert (grads == 0).all()
    P.linear_weight_grad(z(6, 4), z(6, 0, t=torch.int8), z(6), dw[:, :, :0])
    P.linear_weight_grad(z(6, 4) + 2, z(6, 0, t=torch.int8), z(6), grads[:, :0].unflatten(1, (4, 0)), grads[:, 5:9])       # no weight, a bias all the same
    assert (grads[:, 5:9] == 6).all() and (grads[:, :5] == 0).all() and (grads[:, 9:] == 0).all()
    P.linear_weight_grad(z(6, 0), z(6, 3, t=torch.int8), z(6), dw[:, :0])
    assert (dw == 5).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,outs", [(40, 300), (300, 40), (64, 48), (129, 8)])
def test_linear_weight_grad_keeps_24_bits_for_fp32(cols, outs, dtype):
    """Workers of one row: a gradient is one product.  Its factor is rounded to fp32 (2^-24) and cut into planes whose three products are exact; their
    sum is off by at most 2^-23 for each addition, also where it is cut.  Two planes would be off by up to 2^-17."""
    g = gen("weights bits", cols, outs)
    q, scale = Q.quantized(randn(g, 5, cols), False)
    dy = randn(g, 5, outs, std=0.1).to(dtype)
    dw = torch.zeros(5, outs, cols, device="cuda")
    P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), dw)
    want = dy.double()[:, :, None] * (q.double() * scale.double()[:, None])[:, None, :]
    assert ((dw.cpu().double() - want).abs() <= (1 + 2 * 3) * Q.E32 * want.abs() + 2.0 ** -120).all()


@pytest.mark.parametrize("n,per,cols,outs", [(2, 1, 1, 1), (2, 5, 9, 4), (2, 70, 33, 130), (2, 300, 129, 127), (2, 33, 2100, 2080), (2, 4200, 64, 72)])
def test_linear_weight_grad_rows_that_half_precision_does_not_hold(n, per, cols, outs):
    """Scales of 2^-126 to 2^100 beside common ones, a worker with nothing but small ones.

    The sums' tolerance is that of other rows, (per + 64) roundings of 2^-24 of the sum of the products' sizes, but for numbers below half precision's
    least normal one, 2^-14: the matrix unit lines products up by their operands' exponents, which for those is the least normal number's, and cuts them
    24 bits below the largest.  Such a factor counts as 2^-14 in the products' sizes.  An x of up to 2^-25 rounds to zero: it is added apart, in 32 bits."""
    print(f"[case] weights out of half {n}x{per} {cols}->{outs}", flush=True)
    g = gen("weights half", n, per, cols, outs)
    q = whole(g, n * per, cols)
    power = torch.randint(-6, 3, (n * per,), generator=g)
    power[:per] = torch.randint(-60, -24 if per % 2 else -32, (per,), generator=g)         # some and nothing of which rounds to more than zero
    power[0] = -126
    power[-1] = 10
    if per > 30:
        power[per + 7], power[per + 29], power[-2] = 100, -25, -40
    scale = torch.ldexp(torch.ones(n * per), power)
    dy = randn(g, n * per, outs, std=0.1).to(F16)
    dw, db, _, s_db = Q.weight_grad(dy, q, scale, n, True)
    x, d = (q.double() * scale.double()[:, None]).abs().view(n, per, cols), dy.double().abs().view(n, per, outs)
    x = torch.where(x > 2.0 ** -25, x.clamp(min=2.0 ** -14), x)
    s_dw = (d.clamp(min=2.0 ** -14).transpose(1, 2).contiguous() @ x) * ((per + 64) * Q.E32) + 2.0 ** -120
    for pad, lead in ((0, 0), (5, 3)):
        qv, dyv = strided(q, pad, lead)[0], strided(dy, pad, lead, float("nan"))[0]
        for grad in (F32, BF16):
            for turned in (False, True):
                buf = torch.full((n, outs * cols + outs), 7.0, dtype=grad, device="cuda")
                w = buf[:, :outs * cols]
                w = w.unflatten(1, (cols, outs)).transpose(1, 2) if turned else w.unflatten(1, (outs, cols))
                b = buf[:, outs * cols:]
                P.linear_weight_grad(dyv, qv, scale.cuda(), w, b, binary=True)
                R.close(w, dw, s_dw, f"dweight {grad} {turned}")
                R.close(b, db, s_db, "dbias")


def test_linear_weight_grad_half_precision_with_scales_that_are_no_numbers():
    g = gen("weights half nan")
    q, dy = whole(g, 90, 40), randn(g, 90, 48).to(F16)
    scale = torch.ones(90)
    scale[50], scale[20] = float("nan"), 2.0 ** -120
    dw = torch.zeros(3, 48, 40, device="cuda")
    P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), dw, binary=True)
    assert torch.isnan(dw[1]).all() and torch.isfinite(dw[0]).all() and torch.isfinite(dw[2]).all()


def test_linear_weight_grad_infinities_beside_planes_of_the_input():
    """bfloat16, any scales, more outputs than inputs: the second plane of an input that the first one holds is no zero."""
    g = gen("weights inf planes")
    q, scale = Q.quantized(randn(g, 80, 24), True)
    q[q == 0] = 1
    dy = randn(g, 80, 56).to(BF16)
    dy[13, 4], dy[70, 9] = float("inf"), float("-inf")
    dw = torch.zeros(2, 56, 24, device="cuda")
    P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), dw)
    want = torch.einsum("wro,wri->woi", dy.double().view(2, 40, 56), (q.double() * scale.double()[:, None]).view(2, 40, 24))
    got = dw.cpu().double()
    assert not torch.isnan(got).any() and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_weight_grad_infinities_stay_with_their_worker_and_channel(dtype):
    g = gen("weights inf")
    q, scale = Q.quantized(randn(g, 80, 50), True)
    q[q == 0] = 1                                                                  # infinity times zero is no infinity
    for bad in (float("inf"), float("nan")):
        dy = randn(g, 80, 30).to(dtype)
        dy[13, 4] = bad
        for binary in (False, True):
            dw = torch.zeros(2, 30, 50, device="cuda")
            P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), dw, binary=binary)
            want = torch.einsum("wro,wri->woi", dy.double().view(2, 40, 30), (q.double() * scale.double()[:, None]).view(2, 40, 50))
            got = dw.cpu().double()
            assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
            assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
