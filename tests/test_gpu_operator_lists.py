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
