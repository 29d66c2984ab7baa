"""Plain 64-bit forms of the operators on rows in 8 bits and the error bounds that their tests use."""
import torch

import operators_util as R

E32 = 2.0 ** -24
LEAST = 2.0 ** -126
FINITE = {torch.float32: 3.4028234663852886e38, torch.bfloat16: 3.396177326406364e38, torch.float16: 65519.99609375}


def quantized(x, binary, dtype=None):
    """(q, scale) by the definition's own steps in fp32, which both sides round alike; on the CPU."""
    x, finite = x.detach().cpu(), FINITE[dtype or x.dtype]
    x = x.float()
    top = x.abs().amax(-1) if x.shape[-1] else torch.zeros(x.shape[:-1])
    bad = ~torch.isfinite(top)
    s = (torch.where(bad, 0.0, top) / 127).clamp(min=LEAST)
    if binary:
        s = ((s.view(torch.int32) + 0x7FFFFF) & 0x7F800000).view(torch.float32)
    most = torch.where(127 * s <= finite, 127.0, torch.floor(finite / s).clamp(max=126.0))
    q = torch.round(torch.where(bad[..., None], 0.0, x) * (1 / s)[..., None])
    q = torch.minimum(torch.maximum(q, -most[..., None]), most[..., None])
    return q.to(torch.int8), torch.where(bad, float("nan"), s)


def rms(x, residual, gain, eps):
    """(y, h as stored, rstd, slack of y, slack of rstd)"""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    hd = h.double()
    cols = x.shape[-1]
    rstd = 1 / ((hd ** 2).mean(-1) + eps).sqrt()
    y = hd * rstd[:, None] * gain.double()
    # squares are positive: their sum is off by a chain of roundings, its root by half of that; 1/sqrt, the mean's factor: a few more
    rel = (64 + cols / 64) * E32
    return y, h, rstd, y.abs() * (rel + 4 * E32), rstd * rel


def check_q8(q, scale, y, slack, binary, what=""):
    """q, scale against rows y that the kernel knew within slack."""
    q, scale, y, slack = q.cpu().double(), scale.cpu().double(), y.cpu(), slack.cpu()
    top, loose = y.abs().amax(-1), slack.amax(-1)
    want = (top / 127).clamp(min=LEAST)
    off = loose / 127 + 4 * E32 * want
    if binary:
        assert torch.equal(torch.frexp(scale)[0], torch.full_like(scale, 0.5)), f"{what}: scales that are no powers of two"
        assert (scale >= want - off).all() and ((scale / 2 < want + off) | (scale == LEAST)).all(), f"{what}: scale"
    else:
        assert ((scale - want).abs() <= off).all(), f"{what}: scale"
    assert q.abs().max() <= 127
    far = (q * scale[:, None] - y).abs()
    assert (far <= scale[:, None] * (0.5 + 512 * E32) + slack + off[:, None]).all(), f"{what}: values"


def rms_backward(dy, h, rstd, gain, dresidual, n):
    """h: the values that the kept row stands for."""
    dy, h, rstd, gain = (t.double() for t in (dy, h, rstd, gain))
    rows, cols = h.shape
    xh, a = h * rstd[:, None], dy * gain
    along = (a * xh).mean(-1, keepdim=True)
    dx = rstd[:, None] * (a - xh * along)
    past = 0 if dresidual is None else dresidual.double()
    per = rows // n
    dgain = (dy * xh).view(n, per, cols).sum(1)
    chain = 64 + cols / 64
    s_dx = rstd[:, None] * E32 * (6 * a.abs() + xh.abs() * (chain + 8) * (a * xh).abs().mean(-1, keepdim=True)) + 2 * E32 * (dx.abs() + (dx + past).abs())
    s_gain = ((per + 72) * E32 * (dy * xh).abs()).view(n, per, cols).sum(1)
    return dx + past, dgain, s_dx, s_gain


def linear(q, scale, w, wscale, bias):
    """The sums are whole numbers below 2^53: exact in 64 bits."""
    y = (q.double() @ w.double().t()) * scale.double()[:, None] * wscale.double()
    slack = 4 * E32 * y.abs()
    if bias is not None:
        y = y + bias.double()
        slack = slack + 2 * E32 * y.abs()
    return y, slack


def weight_grad(dy, q, scale, n, binary):
    """(dweight [n, outs, cols], dbias [n, outs], their slacks)"""
    rows, outs = dy.shape
    per = rows // n
    x = (q.double() * scale.double()[:, None]).view(n, per, -1)
    d = dy.double().view(n, per, outs)
    dt = d.transpose(1, 2).contiguous()
    size = dt.abs() @ x.abs()
    # 16 bits of mantissa are kept of dy scale (24 of fp32): 2^-17 of each product is lost, nothing of a half-precision number times a power of two
    exact = binary if dy.dtype != torch.float32 else False
    lost = 0 if exact else E32 + (2.0 ** -17 if dy.dtype != torch.float32 else 2.0 ** -24)
    return dt @ x, d.sum(1), size * (lost + (per + 64) * E32) + 2.0 ** -120, d.abs().sum(1) * (per + 64) * E32


close = R.close
