"""The operators of include/comp_ams_operators.h against plain 64-bit forms, through the Python entry points: types, sizes from
one element to long rows, strides, masks that leave a row empty, infinities and NaN, ties, and what must not be touched."""
import math
import zlib

import numpy as np
import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def randn(g, *shape, std=1.0):
    return torch.randn(shape, generator=g) * std


def strided(t, pad_rows=0, lead=0, fill=float("nan")):
    """t's values on the GPU inside a larger array: rows `pad_rows` elements further apart, `lead` elements in front."""
    rows, cols = t.shape
    buf = torch.full((lead + rows * (cols + pad_rows) + 8,), fill, dtype=t.dtype, device="cuda")
    view = buf[lead:lead + rows * (cols + pad_rows)].view(rows, cols + pad_rows)[:, :cols]
    view.copy_(t)
    return view, buf


# --- layer norm ---------------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (3, 2), (5, 7), (4, 16), (9, 33), (2, 64), (7, 130), (3, 255), (3, 256), (6, 257), (5, 511), (5, 512), (4, 768),
              (3, 1023), (3, 1024), (3, 1025), (2, 2047), (2, 2049), (2, 4099), (2, 8192), (2, 8193), (1, 16_385), (1, 33_001), (2, 70_001),
              (1000, 24)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_layer_norm(rows, cols, dtype):
    print(f"[case] norm {rows}x{cols} {dtype}", flush=True)
    g = gen("norm", rows, cols)
    x = (randn(g, rows, cols, std=1.5) + randn(g, rows, 1, std=2.0)).to(dtype)
    gain, shift = randn(g, cols), randn(g, cols)
    xv, _ = strided(x, pad_rows=3, lead=1)
    for sh in (shift, None):
        want = R.norm(x, gain, sh, 1e-5)
        slack = R.norm_slack(x, gain, sh, want[1], want[2])
        out, buf = strided(torch.zeros_like(x), pad_rows=5, lead=3, fill=9.0)
        got = P.layer_norm(xv, gain.cuda(), None if sh is None else sh.cuda(), eps=1e-5, out=out)
        for a, w, s, name in zip(got, want, slack, ("y", "mean", "rstd")):
            R.close(a, w, s, name)
        untouched = torch.ones(buf.numel(), dtype=torch.bool)
        untouched[3:3 + rows * (cols + 5)].view(rows, cols + 5)[:, :cols] = False
        assert (buf.cpu()[untouched] == 9.0).all(), "wrote outside the rows"
    again = P.layer_norm(xv, gain.cuda(), shift.cuda(), out=xv)[0]           # in place
    dense = P.layer_norm(x.cuda(), gain.cuda(), shift.cuda())[0]
    assert R.same_bits(again, dense)


def test_layer_norm_of_leading_dimensions_of_parameters_inside_a_flat_model_and_of_nothing():
    g = gen("norm shape")
    theta = randn(g, 1 + 2 * 37).cuda()
    gain, shift = theta[1:38], theta[38:75]
    x = randn(g, 4, 5, 37).cuda()
    y, mean, rstd = P.layer_norm(x, gain, shift)
    assert y.shape == x.shape and mean.shape == rstd.shape == (4, 5)
    flat = P.layer_norm(x.view(20, 37), gain, shift)
    assert R.same_bits(y.view(20, 37), flat[0]) and R.same_bits(mean.view(20), flat[1])
    y, mean, _ = P.layer_norm(x[:0], gain, shift)
    assert y.shape == (0, 5, 37) and mean.shape == (0, 5)
    one = P.layer_norm(x[0, 0], gain, shift)                                  # one row without leading dimensions
    assert one[1].shape == () and R.same_bits(one[0], flat[0][0])


@pytest.mark.parametrize("dtype", DTYPES)
def test_layer_norm_of_equal_elements_of_large_offsets_and_of_nan(dtype):
    x = torch.zeros(5, 300)
    x[0] = 3.0                                   # no variance: eps alone
    x[1] = 1000.0 + torch.arange(300) % 2        # the mean far above the spread
    x[2, 17] = math.nan
    x[3, 5] = math.inf
    x[4] = torch.linspace(-1, 1, 300)
    x = x.to(dtype)
    gain, shift = torch.ones(300), torch.zeros(300)
    y, mean, rstd = P.layer_norm(x.cuda(), gain.cuda(), shift.cuda(), eps=1e-5)
    want = R.norm(x, gain, shift, 1e-5)
    slack = R.norm_slack(x, gain, shift, want[1], want[2])
    for q in (0, 1, 4):
        R.close(y[q:q + 1], want[0][q:q + 1], slack[0][q:q + 1], f"row {q}")
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all() and not torch.isnan(y[4]).any()


def test_rows_further_apart_than_32_bit_offsets():
    big = torch.empty((3 << 30) + 4096, dtype=torch.bfloat16, device="cuda")
    g = gen("far rows")
    x = randn(g, 3, 600).bfloat16()
    far = big.as_strided((3, 600), (3 << 29, 1))
    far.copy_(x)
    gain, shift = randn(g, 600), randn(g, 600)
    y, mean, rstd = P.layer_norm(far, gain.cuda(), shift.cuda())
    want = R.norm(x, gain, shift, 1e-5)
    R.close(y, want[0], R.norm_slack(x, gain, shift, want[1], want[2])[0], "y")
    dy = randn(g, 3, 600).bfloat16()
    dgain = torch.zeros(1, 600, device="cuda")
    dx = P.layer_norm_backward(dy.cuda(), far, mean, rstd, gain.cuda(), dgain, out=far)
    want = R.norm_backward(dy, x, mean.cpu(), rstd.cpu(), gain, 1)
    R.close(dx, want[0], want[3], "dx")
    R.close(dgain, want[1], want[4], "dgain")
    far.copy_(x)
    logp, entropy, idx, top = P.token_logprobs(far, torch.tensor([5, 0, 599]).cuda(), 4)
    want = R.logprobs(x, torch.tensor([5, 0, 599]), 4)
    assert torch.equal(idx.cpu(), want[2])
    R.close(logp, want[0], want[4], "logp")
    idx, val = torch.tensor([[3, 4], [7, 8], [1, 599]], dtype=torch.int32), randn(g, 3, 2)
    loss, dz = P.distill_grad(far, idx.cuda(), val.cuda(), torch.ones(3).cuda(), out=far)
    want = R.distill(x, idx, val, 1.0, torch.ones(3))
    R.close(loss, want[0], want[3], "loss")
    R.close(dz, want[2], want[5], "dz")
    s = big.as_strided((1, 3, 2, 50), (0, 3 << 29, 900, 1))
    scores = randn(g, 1, 3, 2, 50).bfloat16()
    s.copy_(scores)
    table = randn(g, 3, 3)
    want = R.bias_softmax(scores, table, [-2, 1], 0.5, False, 0, None)
    p = P.rel_bias_softmax(s, table.cuda(), [-2, 1], scale=0.5, out=s)
    R.close(p, want[0], want[1], "p")
    dp = randn(g, 1, 3, 2, 50).bfloat16()
    dtable = torch.zeros(1, 3, 3, device="cuda")
    pc = p.cpu()
    ds = P.rel_bias_softmax_backward(dp.cuda(), p, [-2, 1], dtable, scale=0.5)
    want = R.bias_softmax_backward(dp, pc, [-2, 1], 0.5, False, 0, None, 1)
    R.close(ds, want[0], want[2], "ds")
    R.close(dtable, want[1], want[3], "dtable")


@pytest.mark.parametrize("dtype,grad", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.bfloat16),
                                        (torch.bfloat16, torch.float16)])
@pytest.mark.parametrize("rows,cols,n", [(1, 1, 1), (6, 5, 3), (40, 16, 4), (33, 100, 1), (8, 129, 8), (64, 256, 2), (65, 257, 5), (50, 768, 1),
                                         (300, 512, 3), (12, 1023, 2), (7, 1025, 7), (24, 2047, 4), (9, 4100, 3), (4, 8193, 2), (2, 16_390, 1),
                                         (2, 33_001, 2), (4, 70_001, 2), (5000, 48, 2), (2100, 260, 1)])
def test_layer_norm_backward(rows, cols, n, dtype, grad):
    print(f"[case] norm backward {rows}x{cols} n={n} {dtype} {grad}", flush=True)
    g = gen("norm backward", rows, cols, n)
    x = (randn(g, rows, cols, std=1.5) + randn(g, rows, 1)).to(dtype)
    dy = randn(g, rows, cols, std=0.3).to(dtype)
    gain = randn(g, cols) + 0.5
    _, mean, rstd = (t.float() for t in R.norm(x, gain, None, 1e-5))
    want = R.norm_backward(dy, x, mean, rstd, gain, n)
    grads = torch.full((n, 3 + 2 * cols + 4), 7.0, dtype=grad, device="cuda")
    dgain, dshift = grads[:, 3:3 + cols], grads[:, 3 + cols:3 + 2 * cols]
    xv, _ = strided(x, 1, 3)
    dyv, _ = strided(dy, 2, 5)
    out, _ = strided(torch.zeros_like(x), 4, 1)
    args = (mean.cuda(), rstd.cuda(), gain.cuda())
    dx = P.layer_norm_backward(dyv, xv, *args, dgain, dshift, out=out)
    R.close(dx, want[0], want[3], "dx")
    R.close(dgain, want[1], want[4], "dgain")
    R.close(dshift, want[2], want[5], "dshift")
    host = grads.cpu()
    assert (host[:, :3] == 7).all() and (host[:, 3 + 2 * cols:] == 7).all(), "wrote outside the parameters"
    first = (dx.clone(), grads.clone())
    grads[:, 3:3 + 2 * cols] = 5
    dx = P.layer_norm_backward(dyv, xv, *args, dgain, None, out=dyv)          # in place of dy; no shift
    assert R.same_bits(dx, first[0]) and R.same_bits(dgain, first[1][:, 3:3 + cols]) and (dshift == 5).all()
    dyv.copy_(dy)
    dx = P.layer_norm_backward(dyv, xv, *args, dgain, dshift, out=xv)         # in place of x
    assert R.same_bits(dx, first[0]) and R.same_bits(grads, first[1])


def test_layer_norm_backward_of_no_rows_clears_the_parameter_gradients():
    grads = torch.full((3, 20), 7.0, device="cuda")
    e = torch.empty(0, 8, device="cuda")
    dx = P.layer_norm_backward(e, e, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), torch.ones(8, device="cuda"),
                               grads[:, :8], grads[:, 8:16])
    assert dx.shape == (0, 8) and (grads[:, :16] == 0).all() and (grads[:, 16:] == 7).all()


def test_layer_norm_gradient_against_differences():
    """Central differences of the forward kernel along random directions: sum(y c) moves by 2 h <dx, v> when x moves by +-h v.
    The outputs are off by at most 2^-20 of values up to 8 over 400 elements with random signs, so the quotient by at most
    about 8 * 2^-20 * 20 * 3 / (2 h) = 4e-3 of the sum's scale at h = 0.05; curvature adds h^2 of third derivatives."""
    g = gen("norm differences")
    rows, cols, h = 4, 100, 0.05
    x, c, v = randn(g, rows, cols), randn(g, rows, cols), randn(g, rows, cols)
    gain, shift, gv, sv = randn(g, cols), randn(g, cols), randn(g, cols), randn(g, cols)

    def total(sign):
        y = P.layer_norm((x + sign * h * v).cuda(), (gain + sign * h * gv).cuda(), (shift + sign * h * sv).cuda())[0]
        return float((y.cpu().double() * c.double()).sum())

    _, mean, rstd = P.layer_norm(x.cuda(), gain.cuda(), shift.cuda())
    grads = torch.zeros(1, 2 * cols, device="cuda")
    dx = P.layer_norm_backward(c.cuda(), x.cuda(), mean, rstd, gain.cuda(), grads[:, :cols], grads[:, cols:])
    slope = float((dx.cpu().double() * v).sum() + (grads[0, :cols].cpu().double() * gv).sum() + (grads[0, cols:].cpu().double() * sv).sum())
    scale = float((c.double() ** 2).sum().sqrt())
    assert abs((total(1) - total(-1)) / (2 * h) - slope) < (4e-3 + 10 * h * h) * scale


# --- the biased softmax ---------------------------------------------------------------------------------------------

BIAS_CASES = [
    # batch, heads, tq, tk, causal, offset, lengths, buckets
    (1, 1, 1, 1, False, 0, None, 1),
    (2, 3, 1, 7, True, 6, None, 8),
    (2, 2, 5, 5, True, 0, [5, 0], 8),
    (3, 2, 9, 20, True, 11, [20, 3, 1], 16),
    (2, 1, 17, 17, False, 0, None, 2),
    (1, 2, 33, 64, False, -5, None, 32),
    (2, 2, 40, 100, True, -3, [100, 57], 33),          # the first queries see nothing
    (4, 1, 16, 129, False, 0, [0, 1, 128, 200], 16),   # a length beyond the keys counts as all
    (1, 3, 70, 257, True, 187, None, 64),
    (2, 2, 31, 500, False, 10, [-4, 499], 32),         # a negative length counts as none
    (1, 2, 50, 513, True, 463, None, 128),
    (1, 1, 20, 1025, False, 0, None, 32),
    (1, 2, 130, 2049, True, 1919, None, 32),
    (2, 1, 3, 4097, False, 4000, [4097, 2500], 32),
    (1, 1, 2, 8195, True, 8193, None, 32),
    (1, 1, 3, 20_000, True, 12_000, None, 32),
    (1, 1, 2, 40_001, False, 0, None, 16),
]


def bias_inputs(case, dtype):
    b, h, tq, tk, causal, offset, lens, nb = case
    g = gen("bias", *[str(c) for c in case])
    s = randn(g, b, h, tq, tk, std=6.0).to(dtype)
    bounds = P.rel_bias_bounds(nb, 128, causal)
    assert len(bounds) == nb - 1 and (np.diff(bounds) > 0).all()
    table = randn(g, nb, h, std=2.0)
    return g, s, bounds, table, None if lens is None else torch.tensor(lens, dtype=torch.int32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", BIAS_CASES, ids=lambda c: "x".join(map(str, c[:4])))
def test_rel_bias_softmax(case, dtype):
    print(f"[case] bias {case} {dtype}", flush=True)
    b, h, tq, tk, causal, offset, lens, nb = case
    _, s, bounds, table, ln = bias_inputs(case, dtype)
    vis = R.visible(b, tq, tk, causal, offset, lens).expand_as(s)
    poisoned = torch.where(vis, s, torch.full_like(s, math.nan))              # what is not seen does not matter
    want, slack = R.bias_softmax(s, table, bounds, 0.25, causal, offset, lens)
    kw = dict(scale=0.25, causal=causal, offset=offset, key_lengths=None if ln is None else ln.cuda())
    p = P.rel_bias_softmax(poisoned.cuda(), table.cuda(), bounds, **kw)
    R.close(p, want, slack, "p")
    assert (p.cpu()[~vis] == 0).all()
    # heads beside each other in memory, rows of an odd stride, and in place
    buf = torch.full((b, tq, h, tk + 3), 5.0, dtype=dtype, device="cuda")
    view = buf[..., 1:tk + 1].permute(0, 2, 1, 3)
    view.copy_(s)
    q = P.rel_bias_softmax(view, table.cuda(), bounds, out=view, **kw)
    assert R.same_bits(q, p) and (buf[..., 0] == 5).all() and (buf[..., tk + 1:] == 5).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [40, 300, 1500, 20_000])
def test_rel_bias_softmax_of_infinities_nan_and_lowest_values(width, dtype):
    print(f"[case] bias special {width} {dtype}", flush=True)
    g = gen("bias special", width)
    s = randn(g, 1, 1, 8, width, std=3.0)
    low = float(torch.finfo(dtype).min)
    s[0, 0, 0] = -math.inf                       # nothing left
    s[0, 0, 1, 5:] = -math.inf                   # five left
    s[0, 0, 2] = low                             # all at the type's lowest value: equal scores
    s[0, 0, 3, : width // 2] = low
    s[0, 0, 4, 7] = math.nan
    s[0, 0, 5, 9] = math.inf
    s[0, 0, 6] = 0.0
    s = s.to(dtype)
    table = torch.zeros(1, 1)
    p = P.rel_bias_softmax(s.cuda(), table.cuda(), [], scale=1.0).cpu()
    want, slack = R.bias_softmax(s, table, [], 1.0, False, 0, None)
    assert (p[0, 0, 0] == 0).all()
    assert torch.isnan(p[0, 0, 4]).all() and torch.isnan(p[0, 0, 5]).all()
    for q in (1, 2, 3, 6, 7):
        R.close(p[0, 0, q], want[0, 0, q], slack[0, 0, q], f"row {q}")


@pytest.mark.parametrize("offset", [2 ** 31 - 1, -(2 ** 31) + 1, 100_000, -100_000])
def test_rel_bias_positions_far_outside_the_buckets(offset):
    g = gen("bias offset")
    s, table = randn(g, 1, 2, 3, 70), randn(g, 8, 2)
    bounds = P.rel_bias_bounds(8, 64)
    want, slack = R.bias_softmax(s, table, bounds, 1.0, False, offset, None)
    p = P.rel_bias_softmax(s.cuda(), table.cuda(), bounds, offset=offset)
    R.close(p, want, slack, "p")
    dp, dtable = randn(g, 1, 2, 3, 70), torch.zeros(1, 8, 2, device="cuda")
    ds = P.rel_bias_softmax_backward(dp.cuda(), p, bounds, dtable, offset=offset)
    want = R.bias_softmax_backward(dp, p.cpu(), bounds, 1.0, False, offset, None, 1)
    R.close(ds, want[0], want[2], "ds")
    R.close(dtable, want[1], want[3], "dtable")


def test_bounds_at_the_ends_of_32_bits():
    g = gen("bias bounds")
    s, table = randn(g, 1, 1, 4, 40), randn(g, 4, 1)
    bounds = np.array([-2 ** 31, 2, 2 ** 31 - 1], dtype=np.int32)
    want, slack = R.bias_softmax(s, table, bounds, 1.0, False, 0, None)
    p = P.rel_bias_softmax(s.cuda(), table.cuda(), bounds)
    R.close(p, want, slack, "p")
    dtable = torch.zeros(1, 4, 1, device="cuda")
    dp = randn(g, 1, 1, 4, 40)
    P.rel_bias_softmax_backward(dp.cuda(), p, bounds, dtable)
    want = R.bias_softmax_backward(dp, p.cpu(), bounds, 1.0, False, 0, None, 1)
    R.close(dtable, want[1], want[3], "dtable")


@pytest.mark.parametrize("dtype,grad", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.bfloat16),
                                        (torch.bfloat16, torch.float16)])
@pytest.mark.parametrize("case", BIAS_CASES, ids=lambda c: "x".join(map(str, c[:4])))
def test_rel_bias_softmax_backward(case, dtype, grad):
    print(f"[case] bias backward {case} {dtype} {grad}", flush=True)
    b, h, tq, tk, causal, offset, lens, nb = case
    g, s, bounds, table, ln = bias_inputs(case, dtype)
    p = R.bias_softmax(s, table, bounds, 0.25, causal, offset, lens)[0].to(dtype)
    dp = randn(g, b, h, tq, tk, std=0.5).to(dtype)
    vis = R.visible(b, tq, tk, causal, offset, lens).expand_as(s)
    dp = torch.where(vis & (p != 0), dp, torch.full_like(dp, math.nan))       # no gradient from there, whatever it is
    kw = dict(scale=0.25, causal=causal, offset=offset, key_lengths=None if ln is None else ln.cuda())
    for n in {1, b}:
        want = R.bias_softmax_backward(dp, p, bounds, 0.25, causal, offset, lens, n)
        grads = torch.full((n, 3 + nb * h + 4), 7.0, dtype=grad, device="cuda")
        dtable = grads[:, 3:3 + nb * h].unflatten(1, (nb, h))
        ds = P.rel_bias_softmax_backward(dp.cuda(), p.cuda(), bounds, dtable, **kw)
        R.close(ds, want[0], want[2], "ds")
        R.close(dtable, want[1], want[3], "dtable")
        host = grads.cpu()
        assert (host[:, :3] == 7).all() and (host[:, 3 + nb * h:] == 7).all(), "wrote outside the table"
        buf = torch.full((b, tq, h, tk + 3), 5.0, dtype=dtype, device="cuda")
        view = buf[..., 1:tk + 1].permute(0, 2, 1, 3)
        view.copy_(dp)
        pbuf = torch.full((b, h, tq, tk + 5), math.nan, dtype=dtype, device="cuda")[..., 2:tk + 2]
        pbuf.copy_(p)
        first = grads.clone()
        ds2 = P.rel_bias_softmax_backward(view, pbuf, bounds, dtable, out=view, **kw)
        assert R.same_bits(ds2, ds) and R.same_bits(grads, first) and (buf[..., 0] == 5).all() and (buf[..., tk + 1:] == 5).all()


def test_rel_bias_of_nothing():
    grads = torch.full((2, 3 * 2 + 1), 7.0, device="cuda")
    for shape in ((2, 2, 0, 5), (2, 2, 4, 0), (0, 2, 4, 4)):
        s = torch.zeros(shape, device="cuda")
        assert P.rel_bias_softmax(s, torch.zeros(3, 2, device="cuda"), [0, 1]).shape == shape
        grads.fill_(7.0)
        ds = P.rel_bias_softmax_backward(s, s, [0, 1], grads[:, :6].unflatten(1, (3, 2)))
        assert ds.shape == shape and (grads[:, :6] == 0).all() and (grads[:, 6] == 7).all()


def test_rel_bias_gradient_against_differences():
    """As for the layer norm: sum(p c) along random directions of scores and table, h = 0.02."""
    g = gen("bias differences")
    b, h, t, step = 2, 2, 30, 0.02
    s, c, v = randn(g, b, h, t, t), randn(g, b, h, t, t), randn(g, b, h, t, t)
    bounds = P.rel_bias_bounds(16, 64, True)
    table, tv = randn(g, 16, h), randn(g, 16, h)
    lens = torch.tensor([30, 11], dtype=torch.int32, device="cuda")
    kw = dict(scale=0.7, causal=True, key_lengths=lens)

    def total(sign):
        p = P.rel_bias_softmax((s + sign * step * v).cuda(), (table + sign * step * tv).cuda(), bounds, **kw)
        return float((p.cpu().double() * c.double()).sum())

    p = P.rel_bias_softmax(s.cuda(), table.cuda(), bounds, **kw)
    dtable = torch.zeros(1, 16, h, device="cuda")
    ds = P.rel_bias_softmax_backward(c.cuda(), p, bounds, dtable, **kw)
    slope = float((ds.cpu().double() * v).sum() + (dtable[0].cpu().double() * tv).sum())
    # 120 rows whose probabilities are off by 2^-20 at most, and curvature of order one in each
    assert abs((total(1) - total(-1)) / (2 * step) - slope) < 120 * (2.0 ** -20 / step + 0.5 * step * step)


# --- log probabilities ------------------------------------------------------------------------------------------------

def check_logprobs(z, tokens, k, stride_pad=0):
    want = R.logprobs(z, tokens, k)
    zv, _ = strided(z, stride_pad, 1 if stride_pad else 0)
    logp, entropy, idx, top = P.token_logprobs(zv, tokens.cuda(), k)
    assert torch.equal(idx.cpu(), want[2]), "alternatives"
    R.close(logp, want[0], want[4], "logp")
    R.close(top, want[3], want[4][:, None], "top")
    R.close(entropy, want[1], want[5], "entropy")
    assert idx.dtype == torch.int32 and idx.shape == top.shape == (z.shape[0], k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 2), (4, 9, 9), (5, 100, 20), (2, 127, 127), (3, 300, 128), (2, 1000, 0), (2, 4097, 1),
                                          (3, 8191, 50), (2, 30_001, 20), (2, 32_769, 128), (2, 70_003, 64), (1, 150_000, 100),
                                          (1, 400_001, 33), (300, 777, 5)])
def test_token_logprobs(rows, vocab, k, dtype):
    print(f"[case] logprobs {rows}x{vocab} k={k} {dtype}", flush=True)
    g = gen("logprobs", rows, vocab, k)
    z = randn(g, rows, vocab, std=3.0).to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=g)
    tokens[0] = vocab - 1
    check_logprobs(z, tokens, k, stride_pad=3)


PATTERNS = {
    "equal": lambda v, g: torch.full((v,), 1.5),
    "ascending": lambda v, g: torch.linspace(-9, 9, v),
    "descending": lambda v, g: torch.linspace(9, -9, v),
    "two values": lambda v, g: (torch.arange(v) % 3 == 1).float(),
    "signed zeros": lambda v, g: torch.where(torch.rand(v, generator=g) < 0.5, -0.0, 0.0),
    "one above": lambda v, g: torch.where(torch.arange(v) == v // 2, 60.0, -60.0),
    "banned": lambda v, g: torch.where(torch.rand(v, generator=g) < 0.9, -math.inf, torch.randn(v, generator=g)),
    "five left": lambda v, g: torch.where(torch.arange(v) % (v // 5 + 1) == 3, 1.0, -math.inf),
    "lowest": lambda v, g: torch.where(torch.arange(v) % 7 == 0, torch.randn(v, generator=g), -65504.0),
    # runs of large values at a period at which lanes and vectors repeat
    "period 2048": lambda v, g: torch.where(torch.arange(v) % 2048 < 40, 5.0, 0.0) + 0.001 * torch.arange(v) / v,
    "period 4096": lambda v, g: torch.where(torch.arange(v) % 4096 < 8, 5.0, 0.0) + torch.randn(v, generator=g),
    "period 512": lambda v, g: torch.where(torch.arange(v) % 512 < 2, 5.0, 0.0) + torch.randn(v, generator=g),
    "front": lambda v, g: torch.where(torch.arange(v) < 3000, 5.0, 0.0) + torch.rand(v, generator=g),
    "back": lambda v, g: torch.where(torch.arange(v) >= v - 3000, 5.0, 0.0) + torch.rand(v, generator=g),
}


@pytest.mark.parametrize("vocab", [600, 20_000, 70_000])
@pytest.mark.parametrize("pattern", list(PATTERNS))
@pytest.mark.parametrize("dtype", DTYPES)
def test_token_logprobs_of_ties_orders_and_banned_tokens(pattern, vocab, dtype):
    print(f"[case] logprobs {pattern} {vocab} {dtype}", flush=True)
    g = gen("pattern", pattern, vocab)
    z = torch.stack([PATTERNS[pattern](vocab, g) for _ in range(2)]).to(dtype)
    for k in (1, 16, 128):
        check_logprobs(z, torch.tensor([0, vocab // 2]), k)


@pytest.mark.parametrize("vocab", [400, 40_000, 140_000])
def test_token_logprobs_of_nan_infinities_and_tokens_outside(vocab):
    g = gen("logprobs special", vocab)
    z = randn(g, 6, vocab)
    z[0, 17] = math.nan
    z[0, 300] = math.nan
    z[1, 33] = math.inf
    z[2] = -math.inf
    z[3, 5:] = -math.inf
    check_logprobs(z, torch.tensor([1, 2, 3, 4, -100, vocab]), 10)
    logp, entropy, idx, top = P.token_logprobs(z.cuda(), None, 3)
    assert logp is None and idx[0, :2].tolist() == [17, 300] and int(idx[1, 0]) == 33
    assert P.token_logprobs(z[:0].cuda(), None, 3)[2].shape == (0, 3)


# --- distillation --------------------------------------------------------------------------------------------------------

def lists(g, rows, vocab, k, ragged):
    idx = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).to(torch.int32)
    if ragged:
        many = torch.randint(0, k + 1, (rows, 1), generator=g)
        many[0] = 0                                                          # nothing listed
        idx = torch.where(torch.arange(k) < many, idx, -1)
        idx[-1, -1] = vocab                                                  # outside: not there
    return idx, randn(g, rows, k, std=3.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k,temperature,ragged", [
    (1, 1, 1, 1.0, False), (3, 5, 5, 2.0, True), (4, 100, 20, 0.5, True), (3, 127, 127, 1.0, False), (2, 1000, 128, 4.0, True),
    (5, 4097, 8, 2.0, False), (2, 20_001, 50, 1.0, True), (3, 32_768, 32, 2.0, False), (2, 65_537, 33, 1.0, True),
    (2, 70_001, 100, 3.0, False), (2, 131_073, 16, 1.0, True), (1, 300_001, 128, 2.0, False), (200, 333, 7, 1.0, True)])
def test_distillation(rows, vocab, k, temperature, ragged, dtype):
    print(f"[case] distill {rows}x{vocab} k={k} T={temperature} {dtype}", flush=True)
    g = gen("distill", rows, vocab, k)
    z = randn(g, rows, vocab, std=3.0).to(dtype)
    idx, val = lists(g, rows, vocab, k, ragged)
    weight = torch.rand(rows, generator=g) + 0.1
    want = R.distill(z, idx, val, temperature, weight)
    zv, _ = strided(z, 3, 1)
    ti, tv, w = idx.cuda(), val.cuda(), weight.cuda()
    loss, lse = P.distill(zv, ti, tv, temperature=temperature)
    R.close(loss, want[0], want[3], "loss")
    R.close(lse, want[1], want[4], "lse")
    out, buf = strided(torch.zeros_like(z), 5, 3, fill=9.0)
    dz = P.distill_backward(w, zv, lse, ti, tv, temperature=temperature, out=out)
    R.close(dz, want[2], want[5], "gradient")
    untouched = torch.ones(buf.numel(), dtype=torch.bool)
    untouched[3:3 + rows * (vocab + 5)].view(rows, vocab + 5)[:, :vocab] = False
    assert (buf.cpu()[untouched] == 9).all(), "wrote outside the rows"
    loss2, dz2 = P.distill_grad(zv, ti, tv, w, temperature=temperature)
    R.close(loss2, want[0], want[3], "loss in one pass")
    R.close(dz2, want[2], want[5], "gradient in one pass")
    once = dz2.clone()
    kept = zv.clone()
    loss3, dz3 = P.distill_grad(zv, ti, tv, w, temperature=temperature, out=zv)           # in place
    assert R.same_bits(dz3, once) and R.same_bits(loss3, loss2)
    zv.copy_(kept)
    assert R.same_bits(P.distill_backward(w, zv, lse, ti, tv, temperature=temperature, out=zv), dz)
    if ragged:
        assert float(loss[0]) == 0 and (dz[0] == 0).all() and (dz2[0] == 0).all()


@pytest.mark.parametrize("vocab", [50, 5000, 140_000])
def test_distillation_of_repeated_tokens_certain_teachers_and_banned_tokens(vocab):
    g = gen("distill special", vocab)
    z = randn(g, 5, vocab)
    idx = torch.randint(0, vocab, (5, 6), generator=g).to(torch.int32)
    idx[0] = 7                                                               # one token six times
    idx[1, 1] = idx[1, 4] = idx[1, 0]
    val = randn(g, 5, 6)
    val[2, 1:] = -math.inf                                                   # certain of one token
    val[3] = -1e30
    banned = torch.randint(0, vocab, (20,), generator=g)
    banned = banned[~torch.isin(banned, idx[4].long())]
    z[4, banned] = -math.inf
    w = torch.tensor([1.0, -2.0, 0.5, 0.0, 3.0])
    want = R.distill(z, idx, val, 2.0, w)
    loss, dz = P.distill_grad(z.cuda(), idx.cuda(), val.cuda(), w.cuda(), temperature=2.0)
    R.close(loss, want[0], want[3], "loss")
    R.close(dz, want[2], want[5], "gradient")
    assert (dz[4].cpu()[banned] == 0).all()
    loss2, lse = P.distill(z.cuda(), idx.cuda(), val.cuda(), temperature=2.0)
    R.close(loss2, want[0], want[3], "loss")
    R.close(P.distill_backward(w.cuda(), z.cuda(), lse, idx.cuda(), val.cuda(), temperature=2.0), want[2], want[5], "gradient")
    z[0, 3] = math.nan
    z[1] = -math.inf
    loss, dz = P.distill_grad(z.cuda(), idx.cuda(), val.cuda(), w.cuda(), temperature=2.0)
    assert torch.isnan(loss[:2]).all() and torch.isnan(dz[:2]).all() and not torch.isnan(dz[2:]).any()


def test_distillation_gradient_against_differences():
    """The loss kernel's central differences along a random direction, h = 0.02; losses are off by T^2 2^-24 (16 * 5 + 64) at most."""
    g = gen("distill differences")
    rows, vocab, t, h = 3, 200, 2.0, 0.02
    z, v = randn(g, rows, vocab), randn(g, rows, vocab)
    idx, val = lists(g, rows, vocab, 9, False)
    w = torch.rand(rows, generator=g) + 0.5

    def losses(sign):
        return P.distill((z + sign * h * v).cuda(), idx.cuda(), val.cuda(), temperature=t)[0].cpu().double()

    dz = P.distill_grad(z.cuda(), idx.cuda(), val.cuda(), w.cuda(), temperature=t)[1].cpu().double()
    slope = (losses(1) - losses(-1)) / (2 * h) * w
    assert ((slope - (dz * v).sum(1)).abs() < w * (t * t * 144 * 2.0 ** -24 / h + 4 * h * h)).all()


# --- streams and graphs --------------------------------------------------------------------------------------------------

def everything(d):
    """One call of each operator on the inputs in d; all results in one list."""
    y, mean, rstd = P.layer_norm(d["x"], d["gain"], d["shift"])
    dx = P.layer_norm_backward(d["dy"], d["x"], mean, rstd, d["gain"], d["grads"][:, :96], d["grads"][:, 96:192])
    p = P.rel_bias_softmax(d["s"], d["table"], d["bounds"], scale=0.5, causal=True, key_lengths=d["len"])
    ds = P.rel_bias_softmax_backward(d["dp"], p, d["bounds"], d["grads"][:, 192:216].unflatten(1, (12, 2)), scale=0.5, causal=True,
                                     key_lengths=d["len"])
    logp, entropy, idx, top = P.token_logprobs(d["z"], d["tokens"], 10)
    loss, lse = P.distill(d["student"], idx, top, temperature=2.0)
    dz = P.distill_backward(d["w"], d["student"], lse, idx, top, temperature=2.0)
    loss2, dz2 = P.distill_grad(d["student"], idx, top, d["w"], temperature=2.0)
    return [y, mean, rstd, dx, d["grads"], p, ds, logp, entropy, idx, top, loss, lse, dz, loss2, dz2]


def everything_inputs(seed):
    g = gen("everything", seed)
    d = dict(x=randn(g, 40, 96).bfloat16(), gain=randn(g, 96), shift=randn(g, 96), dy=randn(g, 40, 96).bfloat16(), grads=torch.zeros(4, 220),
             s=randn(g, 4, 2, 20, 20).half(), table=randn(g, 12, 2), dp=randn(g, 4, 2, 20, 20).half(),
             len=torch.tensor([20, 5, 0, 13], dtype=torch.int32), z=randn(g, 12, 140_001).bfloat16(),
             tokens=torch.randint(0, 140_001, (12,), generator=g), student=randn(g, 12, 140_001).bfloat16(), w=torch.rand(12, generator=g))
    d = {k: v.cuda() for k, v in d.items()}
    d["bounds"] = P.rel_bias_bounds(12, 64, True)
    return d


def test_a_recorded_graph_repeats_on_new_inputs_and_results_never_vary():
    d = everything_inputs(0)
    everything(d)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything(d)
    for seed in (1, 2, 3, 1):
        new = everything_inputs(seed)
        for k, v in new.items():
            if k not in ("bounds", "grads"):
                d[k].copy_(v)
        want = [t.clone() for t in everything(new)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert R.same_bits(a, b)
        for a, b in zip(everything(new), want):
            assert R.same_bits(a, b)


def test_a_raw_stream_of_the_callers():
    d = everything_inputs(5)
    want = [t.clone() for t in everything(d)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, mean, rstd = P.layer_norm(d["x"], d["gain"], d["shift"], stream=side.cuda_stream)
    grads = torch.zeros_like(d["grads"])
    side.wait_stream(torch.cuda.current_stream())
    dx = P.layer_norm_backward(d["dy"], d["x"], mean, rstd, d["gain"], grads[:, :96], grads[:, 96:192], stream=side.cuda_stream)
    idx, top = P.token_logprobs(d["z"], None, 10, stream=side.cuda_stream)[2:]
    loss, dz = P.distill_grad(d["student"], idx, top, d["w"], temperature=2.0, stream=side.cuda_stream)
    side.synchronize()
    for a, b in ((y, want[0]), (mean, want[1]), (dx, want[3]), (grads[:, :192], want[4][:, :192]), (idx, want[9]), (top, want[10]), (loss, want[14]),
                 (dz, want[15])):
        assert R.same_bits(a, b)


# --- every shape that holds a row in registers, at sizes that do not fill it ----------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [2050, 6001, 12_001, 16_000, 28_001, 40_001, 60_000, 120_001])
def test_vocabulary_rows_of_every_register_shape(vocab, dtype):
    print(f"[case] vocabulary shape {vocab} {dtype}", flush=True)
    g = gen("vocabulary shape", vocab)
    z = randn(g, 3, vocab, std=3.0).to(dtype)
    check_logprobs(z, torch.randint(0, vocab, (3,), generator=g), 17, stride_pad=1)
    idx, val = lists(g, 3, vocab, 9, False)
    weight = torch.rand(3, generator=g) + 0.1
    want = R.distill(z, idx, val, 2.0, weight)
    zv, _ = strided(z, 1, 0)
    loss, dz = P.distill_grad(zv, idx.cuda(), val.cuda(), weight.cuda(), temperature=2.0)
    R.close(loss, want[0], want[3], "loss")
    R.close(dz, want[2], want[5], "gradient")
    assert R.same_bits(P.distill_grad(zv, idx.cuda(), val.cuda(), weight.cuda(), temperature=2.0, out=zv)[1], dz)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", [(1, 1, 9, 8, False, 0, None, 8), (2, 1, 20, 200, True, 180, [200, 77], 16), (1, 2, 9, 700, False, 3, None, 32),
                                  (2, 1, 5, 1500, True, 1495, [1500, 1000], 32), (1, 1, 6, 3500, True, 3494, None, 32),
                                  (1, 1, 5, 7001, False, 0, [6500], 32), (1, 1, 4, 8192, False, -9, None, 16)],
                         ids=lambda c: "x".join(map(str, c[:4])))
def test_score_rows_of_every_register_shape(case, dtype):
    print(f"[case] score shape {case} {dtype}", flush=True)
    b, h, tq, tk, causal, offset, lens, nb = case
    g, s, bounds, table, ln = bias_inputs(case, dtype)
    kw = dict(scale=0.25, causal=causal, offset=offset, key_lengths=None if ln is None else ln.cuda())
    want, slack = R.bias_softmax(s, table, bounds, 0.25, causal, offset, lens)
    p = P.rel_bias_softmax(s.cuda(), table.cuda(), bounds, **kw)
    R.close(p, want, slack, "p")
    dp = randn(g, b, h, tq, tk, std=0.5).to(dtype)
    back = R.bias_softmax_backward(dp, p.cpu(), bounds, 0.25, causal, offset, lens, 1)
    dtable = torch.zeros(1, nb, h, device="cuda")
    ds = P.rel_bias_softmax_backward(dp.cuda(), p, bounds, dtable, **kw)
    R.close(ds, back[0], back[2], "ds")
    R.close(dtable, back[1], back[3], "dtable")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [20, 200, 400, 1100, 1600, 3001, 5000, 6500, 12_000])
def test_norm_rows_of_every_register_shape(cols, dtype):
    print(f"[case] norm shape {cols} {dtype}", flush=True)
    g = gen("norm shape", cols)
    x, dy = randn(g, 70, cols).to(dtype), randn(g, 70, cols, std=0.3).to(dtype)
    gain = randn(g, cols) + 0.5
    y, mean, rstd = P.layer_norm(x.cuda(), gain.cuda())
    want = R.norm(x, gain, None, 1e-5)
    R.close(y, want[0], R.norm_slack(x, gain, None, want[1], want[2])[0], "y")
    back = R.norm_backward(dy, x, mean.cpu(), rstd.cpu(), gain, 2)
    grads = torch.zeros(2, 2 * cols, device="cuda")
    dx = P.layer_norm_backward(dy.cuda(), x.cuda(), mean, rstd, gain.cuda(), grads[:, :cols], grads[:, cols:])
    R.close(dx, back[0], back[3], "dx")
    R.close(grads[:, :cols], back[1], back[4], "dgain")
    R.close(grads[:, cols:], back[2], back[5], "dshift")
