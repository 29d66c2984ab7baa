"""Products and weight gradients by every tile, whole and in pieces, over sizes that end inside them (tests/rows8_tiles.py): all types of operands and
results, biases, rows apart from each other.  The 64-bit forms are computed on the GPU."""
import zlib

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P
import rows8_tiles as T
import rows8_util as Q

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DTYPES = [F32, BF16, F16]


def generator(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def randn(g, *shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda") * std


def whole(g, *shape):
    return torch.randint(-128, 128, shape, generator=g, dtype=torch.int16, device="cuda").to(torch.int8)


def near(got, want, slack, what):
    """R.close for finite values, without leaving the GPU."""
    off = (got.double() - want).abs() - (2 * R.U[got.dtype] * want.abs() + R.TINY[got.dtype] + slack)
    assert not torch.isnan(off).any() and float(off.max()) <= 0, f"{what}: off by {float(off.max())} too much in {int((off > 0).sum())} of {off.numel()}"


def apart(t, pad, lead, fill):
    """t's values inside a larger array: rows `pad` elements further apart, `lead` in front."""
    rows, cols = t.shape
    view = torch.full((lead + rows * (cols + pad) + 40,), fill, dtype=t.dtype, device="cuda")[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


@pytest.mark.parametrize("size", T.PRODUCTS, ids=str)
def test_products(size):
    rows, cols, outs = size
    print(f"[case] product {size}", flush=True)
    g = generator("product", size)
    q, w = whole(g, rows, cols), whole(g, outs, cols)
    # sums of cols products of 74^2 on average: the results are of the size of 2^6
    s, ws = torch.exp(randn(g, rows) * 0.5) * cols ** -0.5 * 0.02, torch.exp(randn(g, outs) * 0.5) * 0.2
    bias = randn(g, outs, std=20)
    sums = q.double() @ w.double().t().contiguous()
    for b in (None, bias):
        want = sums * s.double()[:, None] * ws.double()
        slack = 4 * Q.E32 * want.abs()
        if b is not None:
            want = want + b.double()
            slack = slack + 2 * Q.E32 * want.abs()
        for dtype in DTYPES:
            for pad, lead in ((0, 0), (16, 32), (3, 1)):
                out = torch.full((rows, outs + 5), 7.0, dtype=dtype, device="cuda")
                P.linear_q8(apart(q, pad, lead, 9), s, apart(w, pad, lead, 9), ws, b, out=out[:, :outs])
                near(out[:, :outs], want, slack, f"{dtype} {pad}")
                assert (out[:, outs:] == 7).all()


@pytest.mark.parametrize("binary", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", T.WEIGHTS, ids=str)
def test_weight_gradients(size, dtype, binary):
    n, per, cols, outs = size
    print(f"[case] weights {size} {dtype} {binary}", flush=True)
    g = generator("weights", size)
    rows = n * per
    q, scale = P.quantize_rows(randn(g, rows, cols) * torch.exp(randn(g, rows, 1) * 0.5), binary=binary)
    dy = randn(g, rows, outs, std=0.1)
    if dtype == F16:
        dy[:, ::3] *= 2.0 ** -16                                      # channels of small gradients
    dy = dy.to(dtype)
    dw, db, s_dw, s_db = Q.weight_grad(dy, q, scale, n, binary)
    for k, grad in enumerate(DTYPES):
        for turned in (False, True):
            pad, lead = ((0, 0), (8, 8), (3, 1))[(k + turned) % 3]
            place = torch.full((n, 3 + outs * cols + outs + 2), 7.0, dtype=grad, device="cuda")
            w = place[:, 3:3 + outs * cols]
            w = w.unflatten(1, (cols, outs)).transpose(1, 2) if turned else w.unflatten(1, (outs, cols))
            b = place[:, 3 + outs * cols:-2]
            P.linear_weight_grad(apart(dy, pad, lead, float("nan")), apart(q, pad, lead, 9), scale, w, b, binary=binary)
            near(w, dw, s_dw, f"dweight {grad} {turned}")
            near(b, db, s_db, f"dbias {grad} {turned}")
            assert (place[:, :3] == 7).all() and (place[:, -2:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [k for k in T.WEIGHTS if T.WEIGHTS[k][0] == 256], ids=str)
def test_infinities_beside_the_largest_tile(size, dtype):
    """An infinity or a NaN in a worker's last row, or in a scale, reaches the gradients that it belongs to, and no others."""
    n, per, cols, outs = size
    print(f"[case] infinities {size} {dtype}", flush=True)
    g = generator("infinities", size)
    rows = n * per
    q = whole(g, rows, cols)
    q[q == 0] = 1                                                     # infinity times zero is no infinity
    scale = torch.ldexp(torch.ones(rows, device="cuda"), torch.randint(-8, 1, (rows,), generator=g, device="cuda"))
    dy = randn(g, rows, outs, std=0.1).to(dtype)
    dy[per - 1, outs - 1], dy[rows - 1, 5] = float("inf"), float("nan")
    for binary in (True, False):
        dw = torch.zeros(n, outs, cols, device="cuda")
        P.linear_weight_grad(dy, q, scale, dw, binary=binary)
        want = torch.zeros_like(dw)
        want[0, outs - 1] = q[per - 1].float() * float("inf")
        want[n - 1, 5] = float("nan")
        assert torch.equal(torch.isnan(dw), torch.isnan(want)) and torch.equal(torch.isinf(dw), torch.isinf(want))
        assert torch.equal(dw[torch.isinf(dw)], want[torch.isinf(want)])
    scale[rows - 1] = float("nan")
    dw = torch.zeros(n, outs, cols, device="cuda")
    P.linear_weight_grad(randn(g, rows, outs, std=0.1).to(dtype), q, scale, dw, binary=True)
    assert torch.isnan(dw[n - 1]).all() and (n == 1 or torch.isfinite(dw[:n - 1]).all())
