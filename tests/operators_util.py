"""Plain 64-bit forms of the operators on the CPU and the error bounds that their tests use."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}      # half a unit, relative, with room for
TINY = {torch.float32: 2.0 ** -125, torch.bfloat16: 2.0 ** -125, torch.float16: 2.0 ** -25}  # one rounding; results below normal range
E32 = 2.0 ** -24


def close(got, want, slack, what=""):
    """|got - want| within one rounding to got's type plus `slack` (an upper bound of the 32-bit arithmetic's error, by element)."""
    got64 = got.detach().cpu().double()
    assert got64.shape == want.shape, (what, got64.shape, want.shape)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got64), nan), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got64[inf], want[inf]), f"{what}: infinities"
    rest = ~(nan | inf)
    tol = (2 * U[got.dtype] * want.abs() + TINY[got.dtype] + slack).expand_as(want)
    bad = (got64 - want).abs()[rest] > tol[rest]
    if bad.any():
        at = torch.nonzero(bad)[0, 0]
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} differ, first got {float(got64[rest][at])} want "
                             f"{float(want[rest][at])} allowed {float(tol[rest][at])}")


def same_bits(a, b):
    view = torch.int16 if a.element_size() == 2 else torch.int32
    return torch.equal(a.contiguous().view(view), b.contiguous().view(view))


# --- layer norm ---------------------------------------------------------------------------------------------------

def norm(x, gain, shift, eps):
    x = x.double()
    mean = x.mean(-1)
    rstd = 1 / (((x - mean[:, None]) ** 2).mean(-1) + eps).sqrt()
    y = (x - mean[:, None]) * rstd[:, None] * gain.double()
    return (y + shift.double() if shift is not None else y), mean, rstd


def norm_slack(x, gain, shift, mean, rstd):
    """Bounds for (y, mean, rstd): the mean is off by a chain of additions, and what is taken from x carries that."""
    chain = 64 + x.shape[1] / 64
    top = x.double().abs().amax(-1)
    m = chain * E32 * top
    spread = (x.double() - mean[:, None]).abs().amax(-1)
    r = rstd * (chain * E32 + 4 * (m + E32 * top) * rstd * (1 + spread * rstd))      # relative: the variance's terms are off by 2 d dm
    y = ((m + 4 * E32 * top) * rstd)[:, None] * gain.double().abs() + (spread * r)[:, None] * gain.double().abs()
    y = y + 4 * E32 * (spread * rstd)[:, None] * gain.double().abs()
    if shift is not None:
        y = y + 2 * E32 * shift.double().abs()
    return y, m, r


def norm_backward(dy, x, mean, rstd, gain, n):
    dy, x, mean, rstd, gain = (t.double() for t in (dy, x, mean, rstd, gain))
    rows, cols = x.shape
    xh = (x - mean[:, None]) * rstd[:, None]
    a = dy * gain
    dx = rstd[:, None] * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
    per = rows // n
    dgain = (dy * xh).view(n, per, cols).sum(1)
    dshift = dy.view(n, per, cols).sum(1)
    chain = 64 + cols / 64
    xe = 4 * E32 * (x.abs() + mean.abs()[:, None]) * rstd.abs()[:, None]             # error of xh
    mean_axh = (a * xh).abs().mean(-1, keepdim=True)
    s_dx = rstd.abs()[:, None] * ((chain * E32) * (a.abs() + a.abs().mean(-1, keepdim=True) + xh.abs() * mean_axh)
                                  + xe * mean_axh + xh.abs() * (a.abs() * xe).mean(-1, keepdim=True))
    add = (per + 64) * E32
    s_g = (add * (dy * xh).abs() + dy.abs() * xe).view(n, per, cols).sum(1)
    s_b = (add * dy.abs()).view(n, per, cols).sum(1)
    return dx, dgain, dshift, s_dx, s_g, s_b


# --- the biased softmax ---------------------------------------------------------------------------------------------

def visible(batch, tq, tk, causal, offset, lens):
    j = torch.arange(tk)
    vis = torch.ones(batch, tq, tk, dtype=torch.bool)
    if causal:
        vis &= (j[None, :] <= torch.arange(tq)[:, None] + offset)[None]
    if lens is not None:
        vis &= (j[None, :] < torch.tensor(lens)[:, None])[:, None, :]
    return vis[:, None]


def buckets(tq, tk, offset, bounds):
    r = torch.arange(tk)[None, :] - torch.arange(tq)[:, None] - offset
    if len(bounds) == 0:
        return torch.zeros(tq, tk, dtype=torch.int64)
    return (r[..., None] >= torch.tensor([int(b) for b in bounds])).sum(-1)


def bias_softmax(s, table, bounds, scale, causal, offset, lens):
    """(probabilities, bound of their 32-bit error)"""
    b, h, tq, tk = s.shape
    vis = visible(b, tq, tk, causal, offset, lens).expand(b, h, tq, tk)
    bias = table.double()[buckets(tq, tk, offset, bounds)].permute(2, 0, 1)
    raw = torch.where(vis, s.double(), 0.0)
    t = raw * scale + bias
    t = torch.where(vis, t, -math.inf)
    top = t.amax(-1, keepdim=True) if tk else t.sum(-1, keepdim=True)
    empty = top == -math.inf
    e = torch.exp(t - torch.where(empty, 0.0, top))
    p = torch.where(empty, 0.0, e / e.sum(-1, keepdim=True))
    p = torch.where(torch.isnan(top), math.nan, p) if tk else p
    # an exponent of size a is off by a few units of a; scores far below the top have p = 0 whatever their size
    near = (t > top - 120)
    a = (torch.where(near & torch.isfinite(raw), (raw * scale).abs(), 0.0) + bias.abs())
    a = torch.where(near, a, 0.0).amax(-1, keepdim=True) if tk else a
    slack = p * E32 * (16 * a + 64 + tk / 64) + 2.0 ** -120
    return p, torch.nan_to_num(slack)


def bias_softmax_backward(dp, p, bounds, scale, causal, offset, lens, n):
    b, h, tq, tk = p.shape
    use = visible(b, tq, tk, causal, offset, lens).expand(b, h, tq, tk) & (p != 0)
    p64 = torch.where(use, p.double(), 0.0)
    d = torch.where(use, dp.double(), 0.0)
    total = (p64 * d).sum(-1, keepdim=True)
    dt = p64 * (d - total)
    index = buckets(tq, tk, offset, bounds).flatten()
    nb = len(bounds) + 1
    size = (p64 * d).abs().sum(-1, keepdim=True)
    s_dt = p64 * E32 * (4 * d.abs() + (64 + tk / 64) * size)

    def table(x):
        out = torch.zeros(b, h, nb, dtype=torch.float64)
        out.index_add_(2, index, x.reshape(b, h, -1))
        return out.view(n, b // n, h, nb).sum(1).transpose(1, 2)
    chain = b // n * tq + tk + 64
    return dt * scale, table(dt), s_dt * abs(scale) + 2 * E32 * (dt * scale).abs(), table(s_dt + chain * E32 * dt.abs())


# --- vocabulary rows ----------------------------------------------------------------------------------------------------

def logprobs(z, tokens, k):
    z = z.double()
    rows, vocab = z.shape
    lse = torch.logsumexp(z, 1)
    bad = torch.isnan(z).any(1) | (z == math.inf).any(1) | (z == -math.inf).all(1)
    lse = torch.where(bad, math.nan, lse)
    lp = z - lse[:, None]
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    entropy = torch.where(bad, math.nan, entropy)
    there = (tokens >= 0) & (tokens < vocab)
    logp = torch.where(there, lp.gather(1, torch.where(there, tokens, 0)[:, None])[:, 0], 0.0)
    key = torch.where(torch.isnan(z), math.inf, z + 0.0)
    # NaN above +infinity: two sorts, the second by whether it is a NaN; both keep the order of equals
    first = torch.sort(key, dim=1, descending=True, stable=True).indices
    isnan = torch.isnan(z).gather(1, first).to(torch.int8)
    idx = first.gather(1, torch.sort(isnan, dim=1, descending=True, stable=True).indices)[:, :k]
    finite = torch.where(torch.isfinite(z), z.abs(), 0.0).amax(1)
    s_lp = E32 * (16 * finite + 64 + vocab / 256)
    return logp, entropy, idx.to(torch.int32), lp.gather(1, idx), s_lp, s_lp * (2 + torch.nan_to_num(entropy))


def teacher(idx, val, vocab, temperature):
    there = (idx >= 0) & (idx < vocab)
    v = torch.where(there, val.double() / temperature, -math.inf)
    q = torch.where(there.any(1, keepdim=True), torch.softmax(v, 1), 0.0)
    return torch.where(there, q, 0.0), there


def distill(z, idx, val, temperature, weight):
    """(loss, lse, gradient, and bounds of their 32-bit errors)"""
    rows, vocab = z.shape
    zt = z.double() / temperature
    lse = torch.logsumexp(zt, 1)
    lp = zt - lse[:, None]
    q, there = teacher(idx, val, vocab, temperature)
    at = torch.where(there, idx, 0).long()
    each = torch.where(q > 0, q * (torch.log(torch.where(q > 0, q, 1.0)) - lp.gather(1, at)), 0.0)
    loss = temperature ** 2 * each.sum(1)
    dense = torch.zeros_like(lp).scatter_add_(1, at, q)
    some = there.any(1)
    w = torch.where(some, weight.double() * temperature, 0.0)[:, None]
    grad = w * (lp.exp() - dense)
    size = torch.where(torch.isfinite(zt), zt.abs(), 0.0).amax(1)
    vsize = torch.where(there & torch.isfinite(val), val.double().abs() / temperature, 0.0).amax(1)
    rel = E32 * (16 * size + 16 * vsize + 64 + vocab / 256)
    s_loss = temperature ** 2 * rel * 4
    s_grad = w.abs() * rel[:, None] * (lp.exp() + dense) + 2.0 ** -120
    return loss, lse, grad, s_loss, rel, s_grad
