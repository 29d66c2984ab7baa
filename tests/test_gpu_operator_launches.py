"""More rows than one launch has workgroups for (2^24 of 256 threads): every row is there, and is what the same call gives for fewer rows."""
import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu
ROWS = (1 << 24) + 4
PART = 1 << 22


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def same_as_in_parts(whole, call):
    """call(lo, hi) gives the rows [lo, hi) of `whole`."""
    for lo in range(0, ROWS, PART):
        hi = min(ROWS, lo + PART)
        for a, b in zip(whole, call(lo, hi)):
            assert R.same_bits(a[lo:hi], b), (lo, hi)


def sums_close(got, want, size, chain):
    """A sum of `chain` terms at most one after the other, `size` the sum of their magnitudes, in 64 bits on the GPU."""
    R.close(got, want.cpu(), (chain * R.E32 * size).cpu(), "sums")


def test_layer_norm_of_many_short_rows():
    x, gain, shift = randn(ROWS, 2, seed=1), randn(2, seed=2), randn(2, seed=3)
    whole = P.layer_norm(x, gain, shift)
    same_as_in_parts(whole, lambda lo, hi: P.layer_norm(x[lo:hi], gain, shift))
    _, mean, rstd = whole
    dy = randn(ROWS, 2, seed=4)
    dgain, dshift = torch.empty(4, 2, device="cuda"), torch.empty(4, 2, device="cuda")
    dx = P.layer_norm_backward(dy, x, mean, rstd, gain, dgain, dshift)
    scratch = torch.empty(1, 2, device="cuda")
    same_as_in_parts([dx], lambda lo, hi: [P.layer_norm_backward(dy[lo:hi], x[lo:hi], mean[lo:hi], rstd[lo:hi], gain, scratch)])
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    chain = ROWS / 4 + 64
    for got, terms in ((dgain, dy.double() * xh), (dshift, dy.double())):
        # an xh is off by a few units of (|x| + |mean|) rstd, which its own size does not bound
        size = (terms.abs() + 8 * dy.double().abs() * (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None] / chain)
        sums_close(got, terms.view(4, -1, 2).sum(1), size.view(4, -1, 2).sum(1), chain)


def test_parameter_gradients_of_more_columns_than_one_launch_joins():
    cols = (1 << 28) + 5
    e, none = torch.empty(0, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda")
    grads = torch.full((1, 2 * cols + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    P.layer_norm_backward(e, e, none, none, torch.ones(cols, device="cuda"), grads[:, :cols], grads[:, cols:2 * cols])
    assert int((grads != 0).sum()) == 1 and float(grads[0, -1]) == 7.0


@pytest.mark.parametrize("tk", [2, 4])          # rows that no lanes hold, and rows of one vector
def test_biased_softmax_of_many_short_rows(tk):
    s, table, bounds = randn(ROWS, 1, 1, tk, seed=5), randn(3, 1, seed=6), [0, 1]
    p = P.rel_bias_softmax(s, table, bounds)
    same_as_in_parts([p], lambda lo, hi: [P.rel_bias_softmax(s[lo:hi], table, bounds)])
    dp = randn(ROWS, 1, 1, tk, seed=7)
    dtable = torch.empty(4, 3, 1, device="cuda")
    ds = P.rel_bias_softmax_backward(dp, p, bounds, dtable)
    scratch = torch.empty(1, 3, 1, device="cuda")
    same_as_in_parts([ds], lambda lo, hi: [P.rel_bias_softmax_backward(dp[lo:hi], p[lo:hi], bounds, scratch)])
    of_key = torch.bucketize(torch.arange(tk, device="cuda"), torch.tensor(bounds, device="cuda"), right=True)
    terms = torch.zeros(4, 3, dtype=torch.float64, device="cuda").index_add_(1, of_key, ds.double().view(4, -1, tk).sum(1))
    size = torch.zeros(4, 3, dtype=torch.float64, device="cuda").index_add_(1, of_key, ds.double().abs().view(4, -1, tk).sum(1))
    sums_close(dtable[:, :, 0], terms, size, ROWS / 4 * tk + 64)


@pytest.mark.parametrize("vocab", [3, 8])
def test_vocabulary_rows_by_the_million(vocab):
    z = randn(ROWS, vocab, seed=8, dtype=torch.bfloat16)
    tokens = torch.arange(ROWS, device="cuda") % vocab
    whole = P.token_logprobs(z, tokens, 2)
    same_as_in_parts(whole, lambda lo, hi: P.token_logprobs(z[lo:hi], tokens[lo:hi], 2))
    idx, val, w = whole[2][:, :1].contiguous(), whole[3][:, :1].contiguous(), randn(ROWS, seed=9)
    loss, lse = P.distill(z, idx, val)
    same_as_in_parts([loss, lse], lambda lo, hi: P.distill(z[lo:hi], idx[lo:hi], val[lo:hi]))
    dz = P.distill_backward(w, z, lse, idx, val)
    same_as_in_parts([dz], lambda lo, hi: [P.distill_backward(w[lo:hi], z[lo:hi], lse[lo:hi], idx[lo:hi], val[lo:hi])])
    both = P.distill_grad(z, idx, val, w)
    same_as_in_parts(both, lambda lo, hi: P.distill_grad(z[lo:hi], idx[lo:hi], val[lo:hi], w[lo:hi]))
