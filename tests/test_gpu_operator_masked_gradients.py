"""Gradients of the biased softmax where dp or p holds infinities or NaN: they stay among the keys that a query sees and gives some
probability to, in the scores' gradient and in the buckets of the table's."""
import math

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P

pytestmark = pytest.mark.gpu


def want(dp, p, bounds, scale, causal, offset, lens):
    """(ds, dtable of one worker, their bounds) in 64 bits: keys that are not seen or have no probability take no part."""
    b, h, tq, tk = p.shape
    use = R.visible(b, tq, tk, causal, offset, lens).expand(b, h, tq, tk) & (p != 0)
    p64, d = torch.where(use, p.double(), 0.0), torch.where(use, dp.double(), 0.0)
    size = torch.where(torch.isfinite(p64 * d), (p64 * d).abs(), 0.0).sum(-1, keepdim=True)
    dt = torch.where(use, p64 * (d - (p64 * d).sum(-1, keepdim=True)), 0.0)
    slack = torch.where(torch.isfinite(dt), p64 * R.E32 * (4 * d.abs() + (64 + tk / 64) * size), 0.0)
    slack = torch.nan_to_num(slack)
    index = R.buckets(tq, tk, offset, bounds).flatten()

    def table(x):
        return torch.zeros(b, h, len(bounds) + 1, dtype=torch.float64).index_add_(2, index, x.reshape(b, h, -1)).sum(0, keepdim=True).transpose(1, 2)
    finite = torch.where(torch.isfinite(dt), dt.abs(), 0.0)
    chain = b * tq + tk + 64
    return dt * scale, table(dt), slack * scale + 2 * R.E32 * finite * scale, table(slack + chain * R.E32 * finite)


WIDTHS = [3, 8, 40, 200, 300, 700, 1500, 3500, 8192, 9001]       # every team of lanes, and rows that none of them holds


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("tk", WIDTHS)
def test_infinities_and_nan_stay_with_the_keys_that_count(tk, causal, dtype):
    print(f"[case] odd gradients {tk} {causal} {dtype}", flush=True)
    g = torch.Generator().manual_seed(tk)
    b, h, tq, nb = 2, 2, 11, 16
    offset, lens = tk - 3, [tk, max(1, tk * 2 // 3)]
    bounds = P.rel_bias_bounds(nb, max(4, tk // 2), causal)
    s = (torch.randn(b, h, tq, tk, generator=g) * 3).to(dtype)
    if tk > 4:
        s[..., 1::3] = -math.inf                                   # seen, and of probability zero
    table = torch.randn(nb, h, generator=g)
    p = R.bias_softmax(s, table, bounds, 0.5, causal, offset, lens)[0].to(dtype)
    dp = (torch.randn(b, h, tq, tk, generator=g) * 0.5).to(dtype)
    dp[..., 1::3] = torch.where(p[..., 1::3] == 0, torch.tensor(math.inf, dtype=dtype), dp[..., 1::3])
    dp[:, 0, 1, 0] = math.inf                                      # at a key that counts
    dp[:, 1, 2, 0] = -math.inf
    dp[:, 0, 4, 0] = math.nan
    p[:, 1, 6, 0] = math.nan
    if dtype != torch.float16:
        dp[:, :, 8] = torch.where(p[:, :, 8] == 0, float(torch.finfo(dtype).max), -3e31)    # dp - total leaves the type where p is zero
    vis = R.visible(b, tq, tk, causal, offset, lens).expand_as(p)
    dp = torch.where(vis, dp, torch.full_like(dp, math.nan))
    ds64, table64, s_ds, s_table = want(dp, p, bounds, 0.5, causal, offset, lens)
    assert torch.isnan(ds64).any() and not torch.isnan(ds64[~vis | (p == 0)]).any()
    dtable = torch.full((1, nb, h), 7.0, device="cuda")
    ds = P.rel_bias_softmax_backward(dp.cuda(), p.cuda(), bounds, dtable, scale=0.5, causal=causal, offset=offset,
                                     key_lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert (ds.cpu()[~vis | (p == 0)] == 0).all()
    R.close(ds, ds64, s_ds, "ds")
    R.close(dtable, table64, s_table, "dtable")
