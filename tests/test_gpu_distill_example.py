"""The distillation example: its gradients per worker against automatic differentiation in 64 bits, and that it learns."""
import pytest
import torch

import paper_2111_00705_amd as P
from paper_2111_00705_amd.examples import distill_workers as D

pytestmark = pytest.mark.gpu


def reference_loss(lay, theta, tokens, lengths, idx, val, bounds):
    """Mean loss of one worker from the definitions, differentiable."""
    batch, length = tokens.shape
    dim = D.WIDTH // D.HEADS
    p = {name: lay.view(theta, name) for name in lay.shape}

    def norm(x, g, b):
        return torch.nn.functional.layer_norm(x, (D.WIDTH,), g, b, 1e-5)

    x0 = p["embed"][tokens.view(-1)]
    qkv = (norm(x0, p["g1"], p["b1"]) @ p["qkv"]).view(batch, length, 3, D.HEADS, dim).permute(2, 0, 3, 1, 4)
    r = torch.arange(length)[None, :] - torch.arange(length)[:, None]
    bucket = (r[..., None] >= torch.tensor([int(b) for b in bounds])).sum(-1)
    s = qkv[0] @ qkv[1].transpose(-1, -2) * dim ** -0.5 + p["bias"][bucket].permute(2, 0, 1)
    seen = (r <= 0) & (torch.arange(length) < lengths[:, None, None])
    probs = torch.softmax(s.masked_fill(~seen[:, None], float("-inf")), -1)
    x1 = x0 + (probs @ qkv[2]).transpose(1, 2).reshape(-1, D.WIDTH) @ p["out"]
    lp = torch.log_softmax(norm(x1, p["g2"], p["b2"]) @ p["head"] / D.TEMPERATURE, -1)
    q = torch.softmax(val.double() / D.TEMPERATURE, -1)
    return (D.TEMPERATURE ** 2 * (q * (q.log() - lp.gather(1, idx.long()))).sum(1)).mean()


def test_gradients_per_worker_of_the_whole_model():
    g = torch.Generator().manual_seed(1)
    lay, n, batch = D.layout(), 3, 2
    theta = torch.randn(lay.d, generator=g) * 0.05
    tokens = torch.randint(0, D.VOCAB, (n, batch, D.LENGTH), generator=g)
    lengths = torch.randint(1, D.LENGTH + 1, (n * batch,), generator=g).to(torch.int32)
    rows = n * batch * D.LENGTH
    idx = torch.stack([torch.randperm(D.VOCAB, generator=g)[:D.TOP] for _ in range(rows)]).to(torch.int32)
    val = torch.randn(rows, D.TOP, generator=g)
    bounds = P.rel_bias_bounds(D.BUCKETS, D.LENGTH, causal=True)
    grads = torch.full((n, lay.d), 3.0, device="cuda")
    loss = D.distill_iteration(P, lay, theta.cuda(), grads, tokens.cuda(), lengths.cuda(), idx.cuda(), val.cuda(), bounds)
    per = batch * D.LENGTH
    for w in range(n):
        th = theta.double().requires_grad_(True)
        want = reference_loss(lay, th, tokens[w], lengths[w * batch:(w + 1) * batch], idx[w * per:(w + 1) * per], val[w * per:(w + 1) * per], bounds)
        want.backward()
        assert abs(float(loss[w]) - float(want.detach())) < 1e-5 * (1 + abs(float(want.detach())))
        got = grads[w].cpu().double()
        for name, (lo, hi) in lay.at.items():
            a, b = got[lo:hi], th.grad[lo:hi]
            # a chain of a dozen 32-bit operators over sums of at most 2000 terms: 1e-4 of the parameter's gradient
            assert float((a - b).norm()) <= 1e-4 * float(b.norm()), (w, name)


def test_the_loss_falls_through_the_compressed_optimiser():
    losses, bits, dense = D.run(iterations=40, n=4, batch=2)
    assert losses[-1] < 0.8 * losses[0] and bits < dense
