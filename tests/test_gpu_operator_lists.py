"""Teacher's lists at the edge: entries of no probability, beside others and alone."""
import math

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("k", [1, 5, 100])
@pytest.mark.parametrize("vocab", [3, 150, 5000, 140_000])
def test_lists_of_nothing_but_minus_infinity(vocab, k, dtype):
    """q = 0 throughout: no loss, and a gradient that moves every token's probability down."""
    g = torch.Generator().manual_seed(vocab + k)
    z = (torch.randn(4, vocab, generator=g) * 2).to(dtype)
    idx = torch.randint(0, vocab, (4, k), generator=g).to(torch.int32)
    val = torch.full((4, k), -math.inf)
    val[1, k // 2] = 1.0                               # one that counts
    idx[2, 0] = -1                                     # one that is not there; with k = 1 the list is empty
    temperature, w = 2.0, torch.tensor([1.0, -0.5, 2.0, 0.25])
    lp = torch.log_softmax(z.double() / temperature, 1)
    q = torch.zeros(4, vocab, dtype=torch.float64)
    q[1, int(idx[1, k // 2])] = 1.0
    some = torch.tensor([True, True, k > 1, True])
    loss = -temperature ** 2 * (q * lp).sum(1)
    grad = (w.double() * temperature * some)[:, None] * (lp.exp() - q)
    rel = R.E32 * (16 * (z.double() / temperature).abs().amax(1) + 64 + vocab / 256)
    ic, vc, wc = idx.cuda(), val.cuda(), w.cuda()
    got, lse = P.distill(z.cuda(), ic, vc, temperature=temperature)
    R.close(got, loss, temperature ** 2 * rel * 4, "loss")
    assert float(got[0]) == 0 and float(got[3]) == 0
    slack = (w.abs().double() * temperature * rel)[:, None] * (lp.exp() + q) + 2.0 ** -120
    R.close(P.distill_backward(wc, z.cuda(), lse, ic, vc, temperature=temperature), grad, slack, "gradient")
    got, dz = P.distill_grad(z.cuda(), ic, vc, wc, temperature=temperature)
    R.close(got, loss, temperature ** 2 * rel * 4, "loss in one pass")
    R.close(dz, grad, slack, "gradient in one pass")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("offset", [-1e4, 3e5, -3e38])
@pytest.mark.parametrize("vocab", [3, 5000, 140_000])
def test_the_teachers_values_count_up_to_a_constant(vocab, offset, dtype):
    """fp32 values hold their distances to the largest exactly, and those decide: bounds in their size, not in that of the values."""
    g = torch.Generator().manual_seed(vocab)
    k, rows, t, w = min(6, vocab), 3, 0.7, torch.tensor([1.0, -0.5, 2.0])
    z = torch.randn(rows, vocab, generator=g).to(dtype)
    idx = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(rows)]).to(torch.int32)
    val = torch.randn(rows, k, generator=g) * 2 + offset           # at -3e38 all equal, and beyond fp32 once divided by T
    dist = (val.double() - val.double().amax(1, keepdim=True)) / t
    logq = dist - dist.exp().sum(1, keepdim=True).log()
    q = logq.exp()
    lp = torch.log_softmax(z.double() / t, 1)
    at = lp.gather(1, idx.long())
    loss = t * t * (q * (logq - at)).sum(1)
    s_q = R.E32 * (8 * dist.abs() + 64)                            # relative
    s_lp = R.E32 * (64 + vocab / 256 + 16 * (z.double() / t).abs().amax(1, keepdim=True))
    s_loss = t * t * (q * (s_q * (1 + logq.abs() + at.abs()) + s_lp)).sum(1)
    dense = torch.zeros_like(lp).scatter_add_(1, idx.long(), q)
    s_dense = torch.zeros_like(lp).scatter_add_(1, idx.long(), q * s_q)
    grad = (w.double() * t)[:, None] * (lp.exp() - dense)
    s_grad = (w.abs().double() * t)[:, None] * (lp.exp() * s_lp + s_dense) + 2.0 ** -120
    ic, vc, wc = idx.cuda(), val.cuda(), w.cuda()
    got, lse = P.distill(z.cuda(), ic, vc, temperature=t)
    R.close(got, loss, s_loss, "loss")
    R.close(P.distill_backward(wc, z.cuda(), lse, ic, vc, temperature=t), grad, s_grad, "gradient")
    got, dz = P.distill_grad(z.cuda(), ic, vc, wc, temperature=t)
    R.close(got, loss, s_loss, "loss in one pass")
    R.close(dz, grad, s_grad, "gradient in one pass")
