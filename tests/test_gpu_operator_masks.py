"""Vocabulary rows in which tokens are masked with large finite numbers, and rows far from zero: the vocabulary's operators against 64-bit
forms.  The bounds grow with the distances to a row's maximum, not with the size of its logits."""
import math

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu
E32 = R.E32


class Want:
    """Everything about logits z [rows, vocab] at a temperature in 64 bits, with bounds of the 32-bit arithmetic's error."""

    def __init__(self, z, temperature=1.0):
        self.t, self.z = temperature, z.double()
        self.top = self.z.amax(1, keepdim=True)
        self.d = (self.z - self.top) / temperature                       # exact distances to the maximum
        self.log_sum = self.d.exp().sum(1, keepdim=True).log()
        self.lp = self.d - self.log_sum
        self.p = self.lp.exp()
        self.entropy = -torch.where(self.p > 0, self.p * self.lp, 0.0).sum(1)
        self.lse = (self.top / temperature + self.log_sum)[:, 0]
        # a distance is off by a few units of itself, its exponential relatively by that; terms below e^-100 add nothing; a thread adds up
        # vocab / 256 terms at most
        self.s_sum = E32 * (8 * self.d.abs().clamp(max=100).amax(1, keepdim=True) + 64 + z.shape[1] / 256)
        self.s_lp = self.s_sum + E32 * (4 * self.d.abs() + 2 * self.lp.abs() + 2 * self.log_sum.abs())

    def distill(self, idx, val, weight):
        """(loss, gradient, their bounds)"""
        there = (idx >= 0) & (idx < self.z.shape[1])
        v = torch.where(there, val.double() / self.t, -math.inf)
        dist = v - v.amax(1, keepdim=True)
        q = torch.softmax(v, 1)
        at = torch.where(there, idx, 0).long()
        lp, s_lp = self.lp.gather(1, at), self.s_lp.gather(1, at)
        size = torch.where(there, v.abs(), 0.0).amax(1, keepdim=True)
        s_q = E32 * (16 * size + 64)                                     # relative
        logq = torch.where(q > 0, q, 1.0).log()
        loss = self.t ** 2 * torch.where(q > 0, q * (logq - lp), 0.0).sum(1)
        s_loss = self.t ** 2 * torch.where(q > 0, q * (s_lp + s_q * (1 + logq.abs() + lp.abs()) + E32 * 16 * dist.abs()), 0.0).sum(1)
        dense = torch.zeros_like(self.lp).scatter_add_(1, at, q)
        w = weight.double()[:, None] * self.t
        grad = w * (self.p - dense)
        s_grad = w.abs() * (self.p * (self.s_sum + E32 * (8 * self.d.abs() + 16)) + dense * (s_q + 16 * E32)) + 2.0 ** -120
        return loss, grad, s_loss, s_grad


def masked(z, how, value):
    """z with `value` in most places; which tokens are left of row 0."""
    vocab = z.shape[1]
    left = torch.zeros(vocab, dtype=torch.bool)
    if how == "prefix":
        left[vocab // 2:] = True
    elif how == "suffix":
        left[:vocab - max(1, min(48, vocab // 2))] = True
    elif how == "all but a few":
        left[torch.linspace(0, vocab - 1, min(100, (vocab + 1) // 2)).long()] = True
    elif how == "all but the end":
        left[vocab - vocab // 8 - 1:] = True
    z = z.clone()
    z[:, ~left] = value
    return z, torch.nonzero(left)[:, 0]


CASES = [(torch.float32, -1e6), (torch.float32, -1e10), (torch.float32, -1e30), (torch.bfloat16, -1e9), (torch.bfloat16, -1e10),
         (torch.float16, -6e4)]
VOCABS = [7, 2048, 4096, 40_003, 140_000]


def lists(g, left, rows, vocab, k):
    k = min(k, left.numel() if left.numel() else vocab)
    pick = torch.stack([torch.randperm(left.numel() if left.numel() else vocab, generator=g)[:k] for _ in range(rows)])
    return (left[pick] if left.numel() else pick).to(torch.int32), torch.randn(rows, k, generator=g) * 2


@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("how", ["prefix", "suffix", "all but a few", "all but the end"])
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype,value", CASES)
def test_distillation_over_tokens_masked_with_a_finite_number(dtype, value, vocab, how, temperature):
    print(f"[case] distill mask {vocab} {how} {value} T={temperature} {dtype}", flush=True)
    g = torch.Generator().manual_seed(vocab)
    z, left = masked((torch.randn(2, vocab, generator=g) * 3).to(dtype), how, value)
    idx, val = lists(g, left, 2, vocab, 9)
    weight = torch.tensor([1.0, 0.3])
    want = Want(z, temperature)
    loss, grad, s_loss, s_grad = want.distill(idx, val, weight)
    zc, ic, vc, wc = z.cuda(), idx.cuda(), val.cuda(), weight.cuda()
    got, lse = P.distill(zc, ic, vc, temperature=temperature)
    R.close(lse, want.lse, want.s_sum[:, 0], "lse")
    R.close(got, loss, s_loss, "loss")
    got, dz = P.distill_grad(zc, ic, vc, wc, temperature=temperature)
    R.close(got, loss, s_loss, "loss in one pass")
    R.close(dz, grad, s_grad, "gradient in one pass")
    # from an lse rounded to 32 bits: a relative error of its last place more
    s_grad = s_grad + want.p * weight.double()[:, None] * temperature * 4 * E32 * (want.lse.abs()[:, None] + want.top.abs() / temperature)
    R.close(P.distill_backward(wc, zc, lse, ic, vc, temperature=temperature), grad, s_grad, "gradient")


@pytest.mark.parametrize("how", ["prefix", "suffix", "all but a few", "all but the end"])
@pytest.mark.parametrize("vocab", VOCABS + [1_100_001])
@pytest.mark.parametrize("dtype,value", CASES)
def test_log_probabilities_over_tokens_masked_with_a_finite_number(dtype, value, vocab, how):
    print(f"[case] logprobs mask {vocab} {how} {value} {dtype}", flush=True)
    g = torch.Generator().manual_seed(vocab + 1)
    z, left = masked((torch.randn(2, vocab, generator=g) * 3).to(dtype), how, value)
    want = Want(z)
    tokens = torch.tensor([int(left[0]), int(left[-1])])
    for k in (0, min(5, left.numel())):
        logp, entropy, idx, top = P.token_logprobs(z.cuda(), tokens.cuda(), k)
        R.close(logp, want.lp.gather(1, tokens[:, None])[:, 0], want.s_lp.gather(1, tokens[:, None])[:, 0], "logp")
        R.close(entropy, want.entropy, want.s_sum[:, 0] * (2 + want.entropy), "entropy")
        best = torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(idx.cpu().long(), best)
        R.close(top, want.lp.gather(1, best), want.s_lp.gather(1, best), "top")


@pytest.mark.parametrize("vocab", VOCABS[1:])
@pytest.mark.parametrize("dtype,value", CASES + [(torch.float32, -3.4028234663852886e38), (torch.float16, -65504.0)])
def test_a_row_of_nothing_but_masked_tokens_is_uniform(dtype, value, vocab):
    z = torch.full((1, vocab), value).to(dtype)
    idx, val = torch.tensor([[vocab // 2, 0]], dtype=torch.int32), torch.tensor([[0.5, -0.5]])
    want = Want(z, 2.0)
    grad, _, s_grad = want.distill(idx, val, torch.ones(1))[1:]
    R.close(P.distill_grad(z.cuda(), idx.cuda(), val.cuda(), torch.ones(1).cuda(), temperature=2.0)[1], grad, s_grad, "gradient")
    entropy = P.token_logprobs(z.cuda(), None, 0)[1]
    R.close(entropy, torch.tensor([math.log(vocab)], dtype=torch.float64), want.s_sum[:, 0] * (2 + math.log(vocab)), "entropy")


@pytest.mark.parametrize("offset", [-1e3, 3e5, -4e6, 1e7])
@pytest.mark.parametrize("vocab", VOCABS)
def test_gradients_and_entropies_of_rows_far_from_zero(vocab, offset):
    """Distances to the maximum are what counts, and fp32 logits hold them exactly."""
    print(f"[case] offset {vocab} {offset}", flush=True)
    g = torch.Generator().manual_seed(vocab + 2)
    z = torch.randn(2, vocab, generator=g) * 3 + offset
    idx, val = lists(g, torch.arange(vocab), 2, vocab, 9)
    for temperature in (1.0, 3.0):
        want = Want(z, temperature)
        grad, _, s_grad = want.distill(idx, val, torch.ones(2))[1:]
        R.close(P.distill_grad(z.cuda(), idx.cuda(), val.cuda(), torch.ones(2).cuda(), temperature=temperature)[1], grad, s_grad, "gradient")
    entropy = P.token_logprobs(z.cuda(), None, 0)[1]
    want = Want(z)
    R.close(entropy, want.entropy, want.s_sum[:, 0] * (2 + want.entropy), "entropy")


def check_logprobs(z, want, k):
    vocab = z.shape[1]
    tokens = torch.tensor([0, vocab - 1])[:z.shape[0]]
    logp, entropy, idx, top = P.token_logprobs(z.cuda(), tokens.cuda(), k)
    R.close(logp, want.lp.gather(1, tokens[:, None])[:, 0], want.s_lp.gather(1, tokens[:, None])[:, 0], "logp")
    R.close(entropy, want.entropy, want.s_sum[:, 0] * (2 + want.entropy), "entropy")
    best = torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(idx.cpu().long(), best)
    R.close(top, want.lp.gather(1, best), want.s_lp.gather(1, best), "top")


@pytest.mark.parametrize("dtype,offset", [(torch.float32, 1e3), (torch.float32, -1e4), (torch.float32, 3e6), (torch.float32, -5e8),
                                          (torch.bfloat16, 300.0), (torch.bfloat16, -1e5), (torch.float16, 2000.0)])
@pytest.mark.parametrize("vocab", VOCABS + [1_100_001])
def test_log_probabilities_and_losses_of_rows_far_from_zero(vocab, dtype, offset):
    print(f"[case] far {vocab} {offset} {dtype}", flush=True)
    g = torch.Generator().manual_seed(vocab + 3)
    z = (torch.randn(2, vocab, generator=g) * 3 * max(1.0, abs(offset) * 2.0 ** -10) + offset).to(dtype)
    check_logprobs(z, Want(z), min(5, vocab))
    idx, val = lists(g, torch.arange(vocab), 2, vocab, 9)
    for temperature in (1.0, 3.0):
        want = Want(z, temperature)
        loss, grad, s_loss, s_grad = want.distill(idx, val, torch.ones(2))
        R.close(P.distill(z.cuda(), idx.cuda(), val.cuda(), temperature=temperature)[0], loss, s_loss, "loss")
        got, dz = P.distill_grad(z.cuda(), idx.cuda(), val.cuda(), torch.ones(2).cuda(), temperature=temperature)
        R.close(got, loss, s_loss, "loss in one pass")
        R.close(dz, grad, s_grad, "gradient in one pass")


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype,value", CASES + [(torch.float32, -3.4028234663852886e38), (torch.bfloat16, float(torch.finfo(torch.bfloat16).min)),
                                                 (torch.float16, -65504.0)])
def test_log_probabilities_and_losses_of_rows_masked_throughout(dtype, value, vocab):
    z = torch.full((1, vocab), value).to(dtype)
    check_logprobs(z, Want(z), min(5, vocab))
    idx, val = torch.tensor([[vocab // 2, 0]], dtype=torch.int32), torch.tensor([[0.5, -0.5]])
    loss, grad, s_loss, s_grad = Want(z, 2.0).distill(idx, val, torch.ones(1))
    R.close(P.distill(z.cuda(), idx.cuda(), val.cuda(), temperature=2.0)[0], loss, s_loss, "loss")
    got, dz = P.distill_grad(z.cuda(), idx.cuda(), val.cuda(), torch.ones(1).cuda(), temperature=2.0)
    R.close(got, loss, s_loss, "loss in one pass")
    R.close(dz, grad, s_grad, "gradient in one pass")


def time_of(call, repeats=7):
    call()
    best = math.inf
    for _ in range(repeats):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("k", [32, 128])
def test_alternatives_of_half_precision_logits_far_from_zero_take_no_longer(k):
    """The bound that a row's k best values reach is as fine as half precision there: rows do not go to the search by bisection, which
    reads them 60 times."""
    g = torch.Generator(device="cuda").manual_seed(k)
    near = torch.randn(1024, 32_000, device="cuda", generator=g) * 2.5
    far = (near + 400.0).half()
    near = near.half()
    idx = P.token_logprobs(far, None, k)[2]
    first = torch.sort(far[:8].cpu().double(), dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(idx[:8].cpu().long(), first)
    assert time_of(lambda: P.token_logprobs(far, None, k)) < 2 * time_of(lambda: P.token_logprobs(near, None, k))
