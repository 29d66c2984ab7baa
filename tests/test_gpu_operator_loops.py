"""The operators at sizes where a team of lanes takes several rows in turn, with the next one on its way, where a workgroup takes its most
queries, and where results leave as a stream: against 64-bit forms on the GPU, and in place."""
import math

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
E32 = R.E32


def close(got, want, slack, what):
    """operators_util.close on the GPU."""
    g = got.double()
    assert g.shape == want.shape, what
    assert torch.equal(torch.isnan(g), torch.isnan(want)), f"{what}: NaN in other places"
    tol = 2 * R.U[got.dtype] * want.abs() + R.TINY[got.dtype] + slack
    bad = (g - want).abs() > tol                                  # false for a NaN
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} differ, first at {torch.nonzero(bad)[0].tolist()}"


def randn(g, *shape, std=1.0):
    return torch.randn(shape, device="cuda", generator=g) * std


def generator(*key):
    return torch.Generator(device="cuda").manual_seed(sum(int(k) * p for k, p in zip(key, (1, 31, 1009, 30011))))


# --- layer norm ---------------------------------------------------------------------------------------------------

# rows of 16 lanes, a wavefront, a workgroup of 256 and of 1024; more than 2048 workgroups' worth.  The last leaves as a stream in any type.
NORM = [(40_000, 40), (40_003, 130), (9000, 700), (8300, 1500), (2500, 5000), (4200, 7001), (2300, 12_000), (12_000, 4100)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", NORM)
def test_layer_norm_with_several_rows_a_team(rows, cols, dtype):
    print(f"[case] norm loop {rows}x{cols} {dtype}", flush=True)
    g = generator(rows, cols)
    x = (randn(g, rows, cols, std=1.5) + randn(g, rows, 1)).to(dtype)
    gain, shift = randn(g, cols) + 0.5, randn(g, cols)
    y, mean, rstd = P.layer_norm(x, gain, shift)
    x64 = x.double()
    m64 = x64.mean(1)
    r64 = 1 / ((x64 - m64[:, None]).square().mean(1) + 1e-5).sqrt()
    chain = (64 + cols / 64) * E32
    s_m = chain * x64.abs().amax(1)
    spread = (x64 - m64[:, None]).abs().amax(1)
    s_r = r64 * (chain + 4 * (s_m + E32 * x64.abs().amax(1)) * r64 * (1 + spread * r64))
    close(mean, m64, s_m, "mean")
    close(rstd, r64, s_r, "rstd")
    s_y = gain.double().abs() * (4 * (s_m + E32 * x64.abs().amax(1)) * r64 + spread * (s_r + 4 * E32 * r64))[:, None] + 2 * E32 * shift.double().abs()
    close(y, (x64 - m64[:, None]) * r64[:, None] * gain.double() + shift.double(), s_y, "y")
    del s_y
    n = 4 if rows % 4 == 0 else 1
    dy = randn(g, rows, cols, std=0.3).to(dtype)
    dgain, dshift = torch.empty(n, cols, device="cuda"), torch.empty(n, cols, device="cuda")
    dx = P.layer_norm_backward(dy, x, mean, rstd, gain, dgain, dshift)
    mu, r = mean.double()[:, None], rstd.double()[:, None]
    xh, a = (x64 - mu) * r, dy.double() * gain.double()
    along = (a * xh).mean(1, keepdim=True)
    e_xh = 4 * E32 * (x64.abs() + mu.abs()) * r
    size = (a * xh).abs().mean(1, keepdim=True)
    s_dx = r * (chain * (a.abs() + a.abs().mean(1, keepdim=True) + xh.abs() * size) + e_xh * size + xh.abs() * (a.abs() * e_xh).mean(1, keepdim=True))
    close(dx, r * (a - a.mean(1, keepdim=True) - xh * along), s_dx, "dx")
    # a team adds up every teams-th row of a chunk, then teams, then chunks by eights: no chain is longer than this
    depth = (32 + rows / n / 256 + 1024 / n / 8 + rows / 1024) * E32
    d64 = dy.double()
    close(dgain, (d64 * xh).view(n, -1, cols).sum(1), (depth * (d64 * xh).abs() + d64.abs() * e_xh).view(n, -1, cols).sum(1), "dgain")
    close(dshift, d64.view(n, -1, cols).sum(1), (depth * d64.abs()).view(n, -1, cols).sum(1), "dshift")
    again = torch.empty_like(dgain)
    assert R.same_bits(P.layer_norm_backward(dy, x, mean, rstd, gain, again, out=dy), dx) and R.same_bits(again, dgain)
    assert R.same_bits(P.layer_norm(x, gain, shift, out=x)[0], y)


# --- the biased softmax ---------------------------------------------------------------------------------------------

def seen(b, tq, tk, causal, offset, lens):
    j = torch.arange(tk, device="cuda")
    vis = torch.ones(1, 1, tq, tk, dtype=torch.bool, device="cuda")
    if causal:
        vis = vis & (j[None, :] <= torch.arange(tq, device="cuda")[:, None] + offset)
    if lens is not None:
        vis = vis & (j[None, :] < lens[:, None])[:, None, None, :]
    return vis.expand(b, 1, tq, tk)


def bucket_of(tq, tk, offset, bounds):
    r = torch.arange(tk, device="cuda")[None, :] - torch.arange(tq, device="cuda")[:, None] - offset
    return torch.bucketize(r, torch.tensor(bounds.tolist(), device="cuda"), right=True)


def lengths(b, tk):
    lens = torch.tensor([1 + (tk * (37 * q + 11) // 97) % tk for q in range(b)], dtype=torch.int32)
    lens[0] = tk
    lens[b // 2] = 0                                   # a sequence without keys between the others
    return lens.cuda()


# batch, heads, tq, tk: teams of 16 lanes, wavefronts over few and over many rows, workgroups; the last leaves as a stream
FORWARD = [(4, 4, 1800, 60), (3, 3, 3001, 250), (2, 8, 600, 300), (8, 16, 520, 133), (2, 4, 1000, 1000), (2, 2, 900, 1500), (2, 3, 700, 4097),
           (3, 16, 1001, 1001)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("b,h,tq,tk", FORWARD)
def test_biased_softmax_with_several_queries_a_team(b, h, tq, tk, causal, dtype):
    print(f"[case] bias loop {b}x{h}x{tq}x{tk} {causal} {dtype}", flush=True)
    g = generator(b, h, tq, tk)
    s = randn(g, b, h, tq, tk, std=6.0)
    s[:, :, 3::17] = -math.inf                         # rows of which nothing is left, between ordinary ones
    s[:, :, 7::29] = float(torch.finfo(dtype).min)     # rows masked throughout
    s[:, :, 11::41, 0] = math.nan
    s[:, :, 12::23, 1:] = -math.inf
    s = s.to(dtype)
    bounds = P.rel_bias_bounds(32, 128, causal)
    table = randn(g, 32, h, std=2.0)
    offset, lens = tk // 2 - tq // 2, lengths(b, tk)
    kw = dict(scale=0.25, causal=causal, offset=offset, key_lengths=lens)
    vis = seen(b, tq, tk, causal, offset, lens)
    p = P.rel_bias_softmax(s.masked_fill(~vis, math.nan), table, bounds, **kw)
    bucket = bucket_of(tq, tk, offset, bounds)
    for q in range(b):
        raw = s[q].double().masked_fill(~vis[q], 0.0) * 0.25
        # a bias beside a score of the type's lowest value is below its last place
        bias = torch.where(raw.abs() > 1e30, 0.0, table.double()[bucket].permute(2, 0, 1))
        t = (raw + bias).masked_fill(~vis[q], -math.inf)
        top = t.amax(-1, keepdim=True)
        want = torch.softmax(torch.where(top == -math.inf, 0.0, t), -1).masked_fill(~vis[q] | (top == -math.inf), 0.0)
        want = torch.where(torch.isnan(top) & vis[q], math.nan, want)
        near = torch.where(t > top - 120, raw.masked_fill(raw.abs() > 1e30, 0.0).abs() + bias.abs(), 0.0).amax(-1, keepdim=True)
        close(p[q], want, torch.nan_to_num(want) * E32 * (16 * near + 64 + tk / 64) + 2.0 ** -120, f"sequence {q}")
    assert R.same_bits(P.rel_bias_softmax(s, table, bounds, out=s, **kw), p)


# batch, heads, tq, tk: enough workgroups for 32 rows a team, and for 16; teams of 16 lanes, a wavefront, a workgroup
BACKWARD = [(6400, 1, 40, 8), (1600, 4, 600, 12), (3200, 1, 300, 20), (6400, 1, 40, 140), (1100, 3, 100, 133), (1600, 4, 40, 530),
            (800, 4, 33, 1030), (110, 30, 40, 1030), (420, 16, 9, 2050)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("b,h,tq,tk", BACKWARD)
def test_biased_softmax_backward_with_many_queries_a_team(b, h, tq, tk, causal, dtype):
    print(f"[case] bias backward loop {b}x{h}x{tq}x{tk} {causal} {dtype}", flush=True)
    g = generator(b, h, tq, tk)
    offset, lens, n = tk // 2 - tq // 2, lengths(b, tk), 2
    bounds = P.rel_bias_bounds(32, 128, causal)
    vis = seen(b, tq, tk, causal, offset, lens)
    p = torch.softmax(randn(g, b, h, tq, tk, std=3.0), -1).masked_fill(~vis, 0.0).to(dtype)
    dp = randn(g, b, h, tq, tk, std=0.5).to(dtype)
    dtable = torch.empty(n, 32, h, device="cuda")
    kw = dict(scale=0.25, causal=causal, offset=offset, key_lengths=lens)
    ds = P.rel_bias_softmax_backward(dp.masked_fill(~vis, math.nan), p, bounds, dtable, **kw)
    index = bucket_of(tq, tk, offset, bounds).flatten()
    want, size, add = (torch.zeros(n, h, 32, dtype=torch.float64, device="cuda") for _ in range(3))
    step = max(1, 30_000_000 // (h * tq * tk))
    for w in range(n):
        for lo in range(w * b // n, (w + 1) * b // n, step):
            hi = min(lo + step, (w + 1) * b // n)
            p64, d64 = p[lo:hi].double(), dp[lo:hi].double()
            dt = p64 * (d64 - (p64 * d64).sum(-1, keepdim=True))
            s_dt = p64 * E32 * (4 * d64.abs() + (64 + tk / 64) * (p64 * d64).abs().sum(-1, keepdim=True))
            close(ds[lo:hi], dt * 0.25, s_dt * 0.25 + 2 * E32 * (dt * 0.25).abs(), f"ds of sequences {lo} to {hi}")
            for to, x in ((want, dt), (size, dt.abs()), (add, s_dt)):
                to[w].index_add_(1, index, x.sum(0).flatten(1))
    # a patch, its patches' places in LDS, the teams, a bucket's places by sixteens, the workgroups' parts by 64
    depth = 64 + (tk + 512) / 16 + 13_000 / (n * h) / 64
    close(dtable, want.transpose(1, 2), (add + depth * E32 * size).transpose(1, 2), "dtable")
    again, inplace = torch.empty_like(dtable), torch.empty_like(dtable)
    plain = P.rel_bias_softmax_backward(dp, p, bounds, again, **kw)             # the zeros of keys that are not seen may have the other sign
    assert torch.equal(plain, ds) and torch.equal(again, dtable)
    assert R.same_bits(P.rel_bias_softmax_backward(dp, p, bounds, inplace, out=dp, **kw), plain) and R.same_bits(inplace, again)


# --- vocabulary rows ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,rows,vocab", [(torch.bfloat16, 4200, 32_800), (torch.float16, 1100, 140_001), (torch.float32, 1100, 70_001),
                                              (torch.float32, 300, 30_001)])
def test_distillation_of_logits_that_come_and_go_as_a_stream(dtype, rows, vocab):
    print(f"[case] distill stream {rows}x{vocab} {dtype}", flush=True)
    g = generator(rows, vocab)
    z = randn(g, rows, vocab, std=2.5).to(dtype)
    idx = torch.randint(0, vocab, (rows, 8), device="cuda", generator=g).to(torch.int32)
    val, w = randn(g, rows, 8), torch.rand(rows, device="cuda", generator=g) + 0.1
    loss, lse = P.distill(z, idx, val, temperature=2.0)
    dz = P.distill_backward(w, z, lse, idx, val, temperature=2.0)
    loss2, dz2 = P.distill_grad(z, idx, val, w, temperature=2.0)
    q = torch.softmax(val.double() / 2, 1)
    for lo in range(0, rows, 256):
        at = slice(lo, min(rows, lo + 256))
        zt = z[at].double() / 2
        lp = torch.log_softmax(zt, 1)
        rel = E32 * (16 * zt.abs().amax(1) + 16 * val[at].double().abs().amax(1) / 2 + 64 + vocab / 256)
        want = 4 * (q[at] * (q[at].log() - lp.gather(1, idx[at].long()))).sum(1)
        close(loss[at], want, 16 * rel, "loss")
        close(loss2[at], want, 16 * rel, "loss in one pass")
        close(lse[at], torch.logsumexp(zt, 1), rel, "lse")
        dense = torch.zeros_like(lp).scatter_add_(1, idx[at].long(), q[at])
        grad = w[at].double()[:, None] * 2 * (lp.exp() - dense)
        slack = w[at].double()[:, None] * 2 * rel[:, None] * (lp.exp() + dense)
        close(dz[at], grad, slack, "gradient")
        close(dz2[at], grad, slack, "gradient in one pass")
    kept = z.clone()
    assert R.same_bits(P.distill_grad(z, idx, val, w, temperature=2.0, out=z)[1], dz2)
    assert R.same_bits(P.distill_backward(w, kept, lse, idx, val, temperature=2.0, out=kept), dz)
