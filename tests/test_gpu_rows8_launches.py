"""Calls of more workgroups than one launch has (2^24 of 256 threads): every row and column is there.  Expected values are formed on the GPU with the
roundings that the operators have, so they are equal."""
import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu
PART = 1 << 26


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def parts(rows):
    for lo in range(0, rows, PART):
        yield lo, min(rows, lo + PART)


@pytest.mark.parametrize("rows,cols", [((1 << 28) + 37, 4), ((1 << 24) + 3, 2)])          # sixteen rows a workgroup, and a workgroup a row
def test_rows_in_8_bits(rows, cols):
    print(f"[case] {rows}x{cols}", flush=True)
    x = torch.randn(rows, cols, device="cuda", generator=gen(1))
    q, scale = P.quantize_rows(x, binary=True)
    for lo, hi in parts(rows):
        a, b = P.quantize_rows(x[lo:hi], binary=True)
        assert torch.equal(q[lo:hi], a) and R.same_bits(scale[lo:hi], b), lo
    assert bool(((q.float() * scale[:, None] - x).abs() <= 0.50001 * scale[:, None]).all())
    x.zero_()
    P.restore_rows(q, scale, out=x)
    for lo, hi in parts(rows):
        assert torch.equal(x[lo:hi], q[lo:hi].float() * scale[lo:hi, None]), lo


def test_norm_of_short_rows_and_gradients_of_many_columns():
    rows = (1 << 24) + 3
    x, gain = torch.randn(rows, 2, device="cuda", generator=gen(2)), torch.randn(2, device="cuda", generator=gen(3))
    y, _, rstd = P.rms_norm(x, gain)
    q, scale, _, _ = P.rms_norm_q8(x, gain)
    for lo, hi in ((0, 1 << 20), (rows - (1 << 20), rows)):
        a, _, r = P.rms_norm(x[lo:hi], gain)
        b, s, _, _ = P.rms_norm_q8(x[lo:hi], gain)
        assert R.same_bits(y[lo:hi], a) and R.same_bits(rstd[lo:hi], r) and torch.equal(q[lo:hi], b) and R.same_bits(scale[lo:hi], s)
    cols = (1 << 29) + 5
    e, none = torch.empty(0, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda")
    grads = torch.full((1, cols + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    P.rms_norm_backward(e, e, none, torch.ones(cols, device="cuda"), grads[:, :cols])
    assert int((grads != 0).sum()) == 1 and float(grads[0, -1]) == 7.0


def test_product_of_a_few_tokens_with_many_channels():
    outs, cols = 140_000_001, 5
    g = gen(4)
    q, s = torch.randint(-128, 128, (2, cols), device="cuda", generator=g, dtype=torch.int16).to(torch.int8), torch.tensor([0.5, 3.0], device="cuda")
    w, ws = torch.empty(outs, cols, dtype=torch.int8, device="cuda"), torch.rand(outs, device="cuda", generator=g)
    w.copy_(torch.arange(outs, device="cuda", dtype=torch.int32)[:, None] * torch.tensor([1, 3, 5, 7, 11], device="cuda", dtype=torch.int32) % 251 - 125)
    y = P.linear_q8(q, s, w, ws, dtype=torch.float32)
    for lo, hi in parts(outs):
        for r in range(2):
            sums = (w[lo:hi].int() * q[r].int()).sum(1).float()
            assert torch.equal(y[r, lo:hi], sums * s[r] * ws[lo:hi]), (r, lo)


@pytest.mark.parametrize("cols", [16, 3])                                            # rows as they stand, and rows that are laid out first
def test_product_of_many_tokens(cols):
    print(f"[case] {cols}", flush=True)
    rows, outs = 1050 << 20, 3
    g = gen(5)
    some = torch.randint(-128, 128, (1 << 20, cols), device="cuda", generator=g, dtype=torch.int16).to(torch.int8)
    q = torch.empty(1050, 1 << 20, cols, dtype=torch.int8, device="cuda")
    q.copy_(some)
    q, s = q.view(rows, cols), torch.rand(rows, device="cuda", generator=g)
    w, ws = torch.randint(-128, 128, (outs, cols), device="cuda", generator=g, dtype=torch.int16).to(torch.int8), torch.rand(outs, device="cuda", generator=g)
    y = P.linear_q8(q, s, w, ws)
    sums = (some.float() @ w.float().t().contiguous())                               # whole numbers below 2^24
    for lo, hi in parts(rows):
        want = (sums.repeat((hi - lo) >> 20, 1) * s[lo:hi, None] * ws).to(torch.bfloat16)
        assert torch.equal(y[lo:hi], want), lo                                        # in value: torch.rand gives zeros, and a bias of zero makes -0 0


def test_weight_gradients_of_the_most_workers():
    n, outs = 65_535, 16_392
    g = gen(6)
    q = torch.randint(-127, 128, (n, 1), device="cuda", generator=g, dtype=torch.int16).to(torch.int8)
    scale = torch.ldexp(torch.ones(n, device="cuda"), torch.randint(-9, 2, (n,), device="cuda", generator=g))
    dy = torch.randn(n, outs, device="cuda", generator=g).to(torch.bfloat16)
    grads = torch.full((n, outs + outs + 2), 7.0, dtype=torch.bfloat16, device="cuda")
    P.linear_weight_grad(dy, q, scale, grads[:, :outs].unflatten(1, (outs, 1)), grads[:, outs:2 * outs], binary=True)
    for lo in range(0, n, 8192):
        at = slice(lo, lo + 8192)
        assert torch.equal(grads[at, :outs], (dy[at].float() * (q[at].float() * scale[at, None])).to(torch.bfloat16)), lo     # in value: sums begin with 0
    assert torch.equal(grads[:, outs:2 * outs], dy) and bool((grads[:, 2 * outs:] == 7).all())


def test_norm_gradients_of_the_most_workers():
    n, cols = 65_535, 40
    g = gen(7)
    h, dy = torch.randn(n * 2, cols, device="cuda", generator=g), torch.randn(n * 2, cols, device="cuda", generator=g)
    rstd, gain = torch.rand(n * 2, device="cuda", generator=g) + 0.5, torch.randn(cols, device="cuda", generator=g)
    dgain = torch.zeros(n, cols, device="cuda")
    P.rms_norm_backward(dy, h, rstd, gain, dgain)
    terms = dy.double() * h.double() * rstd.double()[:, None]
    off = (dgain.double() - terms.view(n, 2, cols).sum(1)).abs()
    assert bool((off <= 6 * R.E32 * terms.abs().view(n, 2, cols).sum(1)).all())      # two roundings a term, one of the sum
