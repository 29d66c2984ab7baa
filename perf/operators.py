"""The operators that a worker's forward and backward pass puts next to the compressed optimiser, as cases that can be
timed and checked: layer norm, the softmax of scores with a learned relative position bias, token log probabilities,
and the distillation loss.

Where `own` is false a pass computes the operator from elementary torch operations in 32 bits, rounded once at the end;
where it is true it makes the calls of the library.  Parameter gradients come per worker: worker w's go to its row of the
optimiser's gradient buffer grads[n, d], at the place where the parameter stands in the flat model.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
LEAD = 5             # parameters that stand before the operator's own in the flat model
TAIL = 6             # and behind it


# --- cases ---------------------------------------------------------------------------------------------------

def _norm(op, rows, cols, dtype, n=1, grad="fp32"):
    return {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "n": n, "grad": grad}


def _bias(op, batch, heads, tq, tk, dtype, causal=False, lengths=False, buckets=32, distance=128, n=1, grad="fp32"):
    return {"op": op, "batch": batch, "heads": heads, "tq": tq, "tk": tk, "dtype": dtype, "causal": causal, "lengths": lengths,
            "buckets": buckets, "distance": distance, "n": n, "grad": grad}


def _probs(rows, vocab, k, dtype, padding=0):
    return {"op": "token_logprobs", "rows": rows, "vocab": vocab, "k": k, "dtype": dtype, "padding": padding}


def _distill(op, rows, vocab, k, dtype, temperature=2.0, ragged=False):
    return {"op": op, "rows": rows, "vocab": vocab, "k": k, "dtype": dtype, "temperature": temperature, "ragged": ragged}


def listed():
    cases = {
        # one new token of a few sequences: nothing but latency
        "norm_few_tokens": _norm("norm", 3, 1024, "bf16"),
        # a BERT-sized layer over the microbatches of eight workers
        "norm_forward_768": _norm("norm", 16_384, 768, "bf16"),
        # its backward pass, gain and shift gradients into eight rows of fp32 gradients
        "norm_backward_768": _norm("norm_backward", 16_384, 768, "bf16", n=8),
        # twenty workers, rows of an odd length that start anywhere, gradients in bfloat16 rows
        "norm_backward_odd": _norm("norm_backward", 20_000, 2047, "fp32", n=20, grad="bf16"),
        # the scores of a BERT-sized layer, padded sequences
        "bias_forward_512": _bias("bias", 16, 12, 512, 512, "bf16", lengths=True),
        # its backward pass, the table's gradient into eight rows
        "bias_backward_512": _bias("bias_backward", 16, 12, 512, 512, "bf16", lengths=True, n=8),
        # a decoder on long sequences of an odd length
        "bias_backward_causal": _bias("bias_backward", 2, 16, 1999, 1999, "f16", causal=True, n=2, grad="f16"),
        # the next token of five sequences with its alternatives: latency
        "logprobs_few_tokens": _probs(5, 32_000, 20, "bf16"),
        # a teacher's record over a batch, a vocabulary padded to a multiple of 32
        "logprobs_teacher": _probs(4096, 100_000, 32, "bf16", padding=17),
        # the student's loss and the gradient of its logits, as a training step calls it
        "distill_step": _distill("distill_grad", 4096, 32_768, 32, "bf16"),
        # the loss alone over a held-out batch, lists cut off at different lengths
        "distill_forward": _distill("distill", 2048, 50_001, 100, "f16", ragged=True),
        # the gradient after a loss whose weights were not known before
        "distill_backward": _distill("distill_backward", 1024, 131_072, 8, "fp32", temperature=1.0),
    }
    return [dict(case, name=name) for name, case in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f16", "fp32"])
    op = rng.choice(["norm", "norm_backward", "bias", "bias_backward", "token_logprobs", "distill", "distill_backward", "distill_grad"])
    n = rng.choice([1, 2, 4, 8, 16, 20])
    grad = rng.choice(["fp32", "bf16", "f16"])
    if op.startswith("norm"):
        cols = _log_int(rng, 32, 8192)
        rows = _log_int(rng, 1, min(65_536, 60_000_000 // cols))
        if op == "norm":
            return _norm(op, rows, cols, dtype)
        return _norm(op, max(n, rows // n * n), cols, dtype, n, grad)
    if op.startswith("bias"):
        heads = rng.choice([1, 4, 8, 12, 16])
        n = rng.choice([1, 2, 4]) if op == "bias_backward" else 1
        if op == "bias" and rng.random() < 0.3:             # one new token against the keys so far
            tq, tk = 1, _log_int(rng, 1, 4096)
        else:
            tq = tk = _log_int(rng, 1, min(4096, int(math.sqrt(60_000_000 / (heads * n)))))
        batch = n * _log_int(rng, 1, max(1, min(64, 60_000_000 // (heads * tq * tk * n))))
        return _bias(op, batch, heads, tq, tk, dtype, rng.random() < 0.5, rng.random() < 0.5, rng.choice([8, 16, 32, 33, 64]),
                     rng.choice([64, 128, 200]), n, grad)
    vocab = _log_int(rng, 300, 150_000)
    rows = _log_int(rng, 1, min(8192, 120_000_000 // vocab))
    k = min(rng.choice([0, 1, 5, 20, 50, 128]), vocab) if op == "token_logprobs" else _log_int(rng, 1, min(128, vocab))
    if op == "token_logprobs":
        return _probs(rows, vocab, k, dtype, rng.choice([0, 0, 1, 63]))
    return _distill(op, rows, vocab, k, dtype, rng.choice([1.0, 2.0, 4.0]), rng.random() < 0.5)


# --- inputs --------------------------------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * int(seed) + 29)
    return gen


def _normal(gen, *shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen)


def _grads(case, size):
    """The optimiser's gradient buffer, and the columns in it that belong to the operator's `size` parameters."""
    buf = torch.zeros((case["n"], LEAD + size + TAIL), dtype=TYPES[case["grad"]], device="cuda")
    return buf[:, LEAD:LEAD + size]


def _widening(many, reach):
    """`many` ascending distances from 1 on: the first half one apart, the others ever wider, the last below `reach`."""
    near = (many + 1) // 2
    at = list(range(1, near + 1))
    for q in range(1, many - near + 1):
        at.append(max(at[-1] + 1, int(near * (reach / near) ** (q / (many - near + 1)))))
    return at


def _bounds(case):
    """Ascending relative positions (key minus query) at which a new bucket begins, one fewer than there are buckets."""
    left = case["buckets"] - 1 if case["causal"] else (case["buckets"] - 1) // 2
    past = [1 - at for at in reversed(_widening(left, case["distance"]))]
    ahead = _widening(case["buckets"] - 1 - left, case["distance"]) if not case["causal"] else []
    return np.array(past + ahead, dtype=np.int32)


def _lengths(case):
    """Keys of each sequence, the same for every seed: one of them empty, one full where there are that many."""
    b, tk = case["batch"], case["tk"]
    lens = [1 + (tk * (37 * q + 11) // 97) % tk for q in range(b)]
    lens[0] = tk
    if b > 2:
        lens[2] = 0
    return lens


def _visible(case):
    """Truth values [batch or 1, 1, tq, tk]."""
    tq, tk = case["tq"], case["tk"]
    j = torch.arange(tk, device="cuda")
    vis = torch.ones((1, 1, tq, tk), dtype=torch.bool, device="cuda")
    if case["causal"]:
        i = torch.arange(tq, device="cuda") + (tk - tq)
        vis = vis & (j[None, :] <= i[:, None])
    if case["lengths"]:
        lens = torch.tensor(_lengths(case), device="cuda")
        vis = vis & (j[None, :] < lens[:, None])[:, None, None, :]
    return vis


def _bucket_index(case):
    tq, tk = case["tq"], case["tk"]
    r = torch.arange(tk, device="cuda")[None, :] - (torch.arange(tq, device="cuda") + (tk - tq))[:, None]
    bounds = torch.tensor(_bounds(case).tolist(), device="cuda")
    return torch.bucketize(r, bounds, right=True)


def _n_buckets(case):
    return len(_bounds(case)) + 1


def _teacher(case, gen):
    """A teacher's lists: k different tokens a row, best first; cut off at any length, even none, where they are ragged."""
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    start = torch.randint(0, vocab, (rows, 1), device="cuda", generator=gen)
    step = torch.randint(0, max(1, vocab // k), (rows, 1), device="cuda", generator=gen) + 1
    step = step.clamp(max=max(1, (vocab - 1) // k))
    at = torch.arange(k, device="cuda")
    idx = ((start + step * at) % vocab).to(torch.int32)
    val = torch.sort(_normal(gen, rows, k, std=2.0), dim=1, descending=True).values.contiguous()
    if case["ragged"]:
        many = torch.randint(0, k + 1, (rows, 1), device="cuda", generator=gen)
        idx = torch.where(at < many, idx, torch.full_like(idx, -1))
    return idx.contiguous(), val


def _inputs(case, seed):
    gen, dtype, op = _generator(seed), TYPES[case["dtype"]], case["op"]
    if op.startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        x = (_normal(gen, rows, cols) * 1.7 + _normal(gen, rows, 1)).to(dtype)
        theta = _normal(gen, LEAD + 2 * cols + TAIL, std=0.2) + 0.6
        s = {"x": x, "gain": theta[LEAD:LEAD + cols], "shift": theta[LEAD + cols:LEAD + 2 * cols]}
        if op == "norm_backward":
            xf = x.double()
            mean = xf.mean(1)
            s["rstd"] = ((xf - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
            s["mean"] = mean.float()
            s["dy"] = _normal(gen, rows, cols, std=0.1).to(dtype)
            place = _grads(case, 2 * cols)
            s["dgain"], s["dshift"] = place[:, :cols], place[:, cols:]
        return s
    if op.startswith("bias"):
        b, h, tq, tk = case["batch"], case["heads"], case["tq"], case["tk"]
        nb = _n_buckets(case)
        theta = _normal(gen, LEAD + nb * h + TAIL)
        s = {"table": theta[LEAD:LEAD + nb * h].view(nb, h), "bounds": _bounds(case), "scale": 0.125, "offset": tk - tq,
             "causal": case["causal"], "len": None}
        if case["lengths"]:
            s["len"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        scores = _normal(gen, b, h, tq, tk, std=8.0)
        if op == "bias":
            s["scores"] = scores.to(dtype)
        else:
            scores = scores.mul_(0.125).masked_fill_(~_visible(case), -math.inf)
            s["probs"] = torch.softmax(scores, -1).nan_to_num_(0.0).to(dtype)
            del scores
            s["dprobs"] = _normal(gen, b, h, tq, tk, std=0.1).to(dtype)
            s["dtable"] = _grads(case, nb * h).unflatten(1, (nb, h))
        return s
    rows, vocab = case["rows"], case["vocab"]
    logits = _normal(gen, rows, vocab, std=2.5).to(dtype)
    s = {"logits": logits}
    if op == "token_logprobs":
        if case["padding"]:
            logits[:, max(1, vocab - case["padding"]):] = -math.inf       # columns that no token has
        s["tokens"] = torch.randint(0, max(1, vocab - case["padding"]), (rows,), device="cuda", generator=gen)
        s["k"] = case["k"]
        return s
    s["idx"], s["val"] = _teacher(case, gen)
    s["temperature"] = case["temperature"]
    s["weight"] = torch.rand(rows, device="cuda", generator=gen) / rows
    if op == "distill_backward":
        s["lse"] = torch.cat([torch.logsumexp(c.double() / case["temperature"], 1) for c in logits.split(256)]).float()
    return s


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if not own and case["op"].startswith("bias"):
        # what does not change from call to call is laid out once: which table row each place takes, which places count
        state["bucket"] = _bucket_index(case)
        state["visible"] = _visible(case)
        # of the relative positions from the last query's first key to the first query's last key: which bucket has each
        along = torch.cat([state["bucket"].flip(0)[:, 0], state["bucket"][0, 1:]])
        state["member"] = (along[:, None] == torch.arange(_n_buckets(case), device="cuda")).float()
    return state


# --- the plain forms -----------------------------------------------------------------------------------------

def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = torch.rsqrt((xc * xc).mean(1) + EPS)
    y = xc * rstd[:, None] * s["gain"] + s["shift"]
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_norm_backward(s):
    n, cols = s["dgain"].shape
    x, dy = s["x"].float(), s["dy"].float()
    xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
    a = dy * s["gain"]
    dx = s["rstd"][:, None] * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    s["dgain"].copy_((dy * xh).view(n, -1, cols).sum(1))
    s["dshift"].copy_(dy.view(n, -1, cols).sum(1))
    return {"dx": dx.to(s["x"].dtype), "dgain": s["dgain"], "dshift": s["dshift"]}


def _plain_bias(s):
    t = s["scores"].float() * s["scale"] + s["table"][s["bucket"]].permute(2, 0, 1)
    t = torch.where(s["visible"], t, -math.inf)
    top = t.amax(-1, keepdim=True)
    e = torch.exp(t - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    return (e / torch.where(total == 0, 1.0, total)).to(s["scores"].dtype)


def _plain_bias_backward(s):
    p = s["probs"].float()
    d = torch.where(p == 0, 0.0, s["dprobs"].float())
    dt = p * (d - (p * d).sum(-1, keepdim=True))
    n, nb, h = s["dtable"].shape
    per = dt.view(n, -1, *dt.shape[1:]).sum(1)                             # [n, h, tq, tk]
    tq, tk = per.shape[2:]
    # queries turned round and every row one place further: a relative position becomes a column
    per = torch.nn.functional.pad(per.flip(2), (0, tq)).flatten(2)[:, :, :-tq].view(n, h, tq, tk + tq - 1).sum(2)
    s["dtable"].copy_((per @ s["member"]).transpose(1, 2))
    return {"dscores": (dt * s["scale"]).to(s["probs"].dtype), "dtable": s["dtable"]}


def _plain_token_logprobs(s):
    z = s["logits"].float()
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1)
    lse = top[:, 0] + torch.log(total)
    entropy = lse - torch.where(e > 0, e * z, 0.0).sum(1) / total
    del e
    logp = z.gather(1, s["tokens"][:, None])[:, 0] - lse
    # the lower index first among equals: one whole number per place, the value's order above, the index below
    bits = (z + 0.0).view(torch.int32)
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).to(torch.int64)
    place = torch.arange(z.shape[1], device=z.device)
    keys = (order << 32) + (0x7FFFFFFF - place)
    idx = 0x7FFFFFFF - (torch.topk(keys, s["k"], dim=1).values & 0x7FFFFFFF)
    return {"logp": logp, "entropy": entropy, "idx": idx.to(torch.int32), "top": z.gather(1, idx) - lse[:, None]}


def _plain_teacher(s):
    """(shares q of the listed tokens, which are listed, their places)"""
    vocab = s["logits"].shape[1]
    there = (s["idx"] >= 0) & (s["idx"] < vocab)
    v = torch.where(there, s["val"] / s["temperature"], -math.inf)
    top = v.amax(1, keepdim=True)
    e = torch.exp(v - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(1, keepdim=True)
    q = e / torch.where(total == 0, 1.0, total)
    return q, there, torch.where(there, s["idx"], 0).long()


def _plain_lse(z):
    top = z.amax(1, keepdim=True)
    return (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]


def _plain_loss(s, z, lse, q, there, at):
    lp = z.gather(1, at) - lse[:, None]
    logq = torch.log(torch.where(q > 0, q, 1.0))
    return s["temperature"] ** 2 * torch.where(q > 0, q * (logq - lp), 0.0).sum(1)


def _plain_gradient(s, z, lse, q, there, at, weight):
    p = torch.exp(z - lse[:, None])
    p = torch.where(there.any(1, keepdim=True), p, 0.0)
    p.scatter_add_(1, at, -q)
    return (p * (weight * s["temperature"])[:, None]).to(s["logits"].dtype)


def _plain_distill(s):
    z = s["logits"].float() / s["temperature"]
    lse = _plain_lse(z)
    return {"loss": _plain_loss(s, z, lse, *_plain_teacher(s)), "lse": lse}


def _plain_distill_backward(s):
    z = s["logits"].float() / s["temperature"]
    return _plain_gradient(s, z, s["lse"], *_plain_teacher(s), s["weight"])


def _plain_distill_grad(s):
    z = s["logits"].float() / s["temperature"]
    lse = _plain_lse(z)
    teacher = _plain_teacher(s)
    return {"loss": _plain_loss(s, z, lse, *teacher), "dlogits": _plain_gradient(s, z, lse, *teacher, s["weight"])}


PLAIN = {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "bias": _plain_bias, "bias_backward": _plain_bias_backward,
         "token_logprobs": _plain_token_logprobs, "distill": _plain_distill, "distill_backward": _plain_distill_backward,
         "distill_grad": _plain_distill_grad}


def run(state):
    op = state["case"]["op"]
    if not own:
        return PLAIN[op](state)
    import paper_2111_00705_amd as P
    s = state
    if op == "norm":
        y, mean, rstd = P.layer_norm(s["x"], s["gain"], s["shift"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_backward":
        dx = P.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gain"], s["dgain"], s["dshift"])
        return {"dx": dx, "dgain": s["dgain"], "dshift": s["dshift"]}
    if op == "bias":
        return P.rel_bias_softmax(s["scores"], s["table"], s["bounds"], scale=s["scale"], causal=s["causal"], offset=s["offset"],
                                  key_lengths=s["len"])
    if op == "bias_backward":
        dscores = P.rel_bias_softmax_backward(s["dprobs"], s["probs"], s["bounds"], s["dtable"], scale=s["scale"], causal=s["causal"],
                                              offset=s["offset"], key_lengths=s["len"])
        return {"dscores": dscores, "dtable": s["dtable"]}
    if op == "token_logprobs":
        logp, entropy, idx, top = P.token_logprobs(s["logits"], s["tokens"], s["k"])
        return {"logp": logp, "entropy": entropy, "idx": idx, "top": top}
    if op == "distill":
        loss, lse = P.distill(s["logits"], s["idx"], s["val"], temperature=s["temperature"])
        return {"loss": loss, "lse": lse}
    if op == "distill_backward":
        return P.distill_backward(s["weight"], s["logits"], s["lse"], s["idx"], s["val"], temperature=s["temperature"])
    loss, dlogits = P.distill_grad(s["logits"], s["idx"], s["val"], s["weight"], temperature=s["temperature"])
    return {"loss": loss, "dlogits": dlogits}


# --- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    op, es = case["op"], SIZE[case["dtype"]]
    if op.startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        if op == "norm":
            return {"bytes": 2 * es * rows * cols + 8 * cols + 8 * rows, "flops": 8 * rows * cols}
        return {"bytes": 3 * es * rows * cols + 8 * rows + 4 * cols + 2 * case["n"] * cols * SIZE[case["grad"]],
                "flops": 14 * rows * cols}
    if op.startswith("bias"):
        b, h, tq, tk = case["batch"], case["heads"], case["tq"], case["tk"]
        lens = _lengths(case) if case["lengths"] else [tk] * b
        seen = 0
        for n in lens:
            if case["causal"]:
                seen += sum(min(n, tk - tq + i + 1) for i in range(tq))
            else:
                seen += n * tq
        table = _n_buckets(case) * h
        if op == "bias":
            return {"bytes": es * h * (seen + b * tq * tk) + 4 * table, "flops": 8 * h * seen}
        return {"bytes": es * h * (2 * seen + b * tq * tk) + case["n"] * table * SIZE[case["grad"]], "flops": 7 * h * seen}
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    cells = rows * vocab
    if op == "token_logprobs":
        return {"bytes": es * cells + rows * (8 + 8 + 8 * k), "flops": 6 * cells}
    lists = rows * 8 * k
    if op == "distill":
        return {"bytes": es * cells + lists + 8 * rows, "flops": 4 * cells}
    if op == "distill_backward":
        return {"bytes": 2 * es * cells + lists + 8 * rows, "flops": 4 * cells}
    return {"bytes": 2 * es * cells + lists + 8 * rows, "flops": 7 * cells}


# --- the same from the definitions, in 64 bits ---------------------------------------------------------------

def _parts(total, cells_per_row, most=40_000_000):
    """Row ranges small enough for 64-bit copies."""
    step = max(1, most // max(1, cells_per_row))
    return [(lo, min(total, lo + step)) for lo in range(0, total, step)]


def _exact_norm(case, s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, dim=1, unbiased=False)
    rstd = 1.0 / torch.sqrt(var + EPS)
    y = torch.addcmul(s["shift"].double(), (x - mean.unsqueeze(1)) * rstd.unsqueeze(1), s["gain"].double())
    return {"y": y, "mean": mean, "rstd": rstd}


def _exact_norm_backward(case, s):
    """The Jacobian of a normalised row applied to the gradient, one worker after the other."""
    n, cols = case["n"], case["cols"]
    per = case["rows"] // n
    dx, dgain, dshift = [], [], []
    for w in range(n):
        at = slice(w * per, (w + 1) * per)
        r = s["rstd"][at].double()
        unit = (s["x"][at].double() - s["mean"][at].double().unsqueeze(1)) * r.unsqueeze(1)
        up = s["dy"][at].double()
        dgain.append(torch.einsum("rc,rc->c", up, unit))
        dshift.append(up.sum(0))
        inner = up * s["gain"].double()
        along = torch.einsum("rc,rc->r", inner, unit) / cols
        dx.append((inner - inner.sum(1, keepdim=True) / cols - along.unsqueeze(1) * unit) * r.unsqueeze(1))
    return {"dx": torch.cat(dx), "dgain": torch.stack(dgain), "dshift": torch.stack(dshift)}


def _exact_rows(case):
    """For every query: (table row of every key, which keys the sequence length leaves are also allowed by position)."""
    tq, tk = case["tq"], case["tk"]
    bounds = torch.tensor(_bounds(case).tolist(), device="cuda")
    key = torch.arange(tk, device="cuda")
    for i in range(tq):
        r = key - (i + tk - tq)
        yield i, (r[:, None] >= bounds[None, :]).sum(1), (r <= 0) if case["causal"] else torch.ones_like(r, dtype=torch.bool)


def _exact_bias(case, s):
    b, h, tq, tk = s["scores"].shape
    out = torch.zeros((b, h, tq, tk), dtype=torch.float64, device="cuda")
    lens = torch.tensor(_lengths(case) if case["lengths"] else [tk] * b, device="cuda")
    table = s["table"].double()
    key = torch.arange(tk, device="cuda")
    for i, bucket, allowed in _exact_rows(case):
        t = s["scores"][:, :, i].double() * s["scale"] + table[bucket].t()
        use = (allowed & (key < lens[:, None]))[:, None, :].expand(b, h, tk)
        out[:, :, i] = torch.softmax(t.masked_fill(~use, -math.inf), -1).masked_fill(~use, 0.0)
    return out


def _exact_bias_backward(case, s):
    b, h, tq, tk = s["probs"].shape
    n, nb = case["n"], _n_buckets(case)
    ds = torch.empty((b, h, tq, tk), dtype=torch.float64, device="cuda")
    onehot = torch.zeros((tk, nb), dtype=torch.float64, device="cuda")
    table = torch.zeros((b * h, nb), dtype=torch.float64, device="cuda")
    for i, bucket, _ in _exact_rows(case):
        p = s["probs"][:, :, i].double()
        d = s["dprobs"][:, :, i].double()
        dt = p * d - p * (p * d).sum(-1, keepdim=True)
        ds[:, :, i] = dt * s["scale"]
        onehot.zero_()
        onehot[torch.arange(tk, device="cuda"), bucket] = 1.0
        table += dt.reshape(b * h, tk) @ onehot
    return {"dscores": ds, "dtable": table.view(n, b // n, h, nb).sum(1).transpose(1, 2).contiguous()}


def _exact_token_logprobs(case, s):
    outs = []
    for lo, hi in _parts(case["rows"], case["vocab"]):
        z = s["logits"][lo:hi].double()
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        logp = lp[torch.arange(hi - lo, device="cuda"), s["tokens"][lo:hi]]
        entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
        order = torch.sort(z + 0.0, dim=1, descending=True, stable=True).indices[:, :case["k"]]
        outs.append((logp, entropy, order.to(torch.int32), lp.gather(1, order)))
    return dict(zip(("logp", "entropy", "idx", "top"), (torch.cat(o) for o in zip(*outs))))


def _exact_distill_part(case, s, lo, hi):
    """(log probabilities at the temperature, dense teacher distribution with zeros outside its list, lse)"""
    temp, vocab, rows = case["temperature"], case["vocab"], hi - lo
    z = s["logits"][lo:hi].double() / temp
    lse = torch.logsumexp(z, 1)
    idx, val = s["idx"][lo:hi].long(), s["val"][lo:hi].double() / temp
    there = (idx >= 0) & (idx < vocab)
    q = torch.softmax(val.masked_fill(~there, -math.inf), 1).masked_fill(~there, 0.0)
    dense = torch.zeros((rows, vocab + 1), dtype=torch.float64, device="cuda")
    dense.scatter_add_(1, torch.where(there, idx, vocab), q)
    return z - lse[:, None], dense[:, :vocab], lse, q, there


def _exact_distill(case, s, want):
    outs = []
    temp = case["temperature"]
    for lo, hi in _parts(case["rows"], case["vocab"]):
        lp, dense, lse, q, there = _exact_distill_part(case, s, lo, hi)
        loss = temp * temp * (torch.special.xlogy(q, q).sum(1) - torch.where(dense > 0, dense * lp, torch.zeros_like(lp)).sum(1))
        part = [loss, lse]
        if want != "distill":
            if want == "distill_backward":
                lp = s["logits"][lo:hi].double() / temp - s["lse"][lo:hi].double()[:, None]
            grad = lp.exp().sub_(dense).mul_((s["weight"][lo:hi].double() * temp)[:, None])
            part.append(grad.masked_fill_(~there.any(1, keepdim=True), 0.0))
        outs.append(part)
    outs = [torch.cat(o) for o in zip(*outs)]
    if want == "distill":
        return {"loss": outs[0], "lse": outs[1]}
    return outs[2] if want == "distill_backward" else {"loss": outs[0], "dlogits": outs[2]}


def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op in ("distill", "distill_backward", "distill_grad"):
        return _exact_distill(case, s, op)
    return {"norm": _exact_norm, "norm_backward": _exact_norm_backward, "bias": _exact_bias, "bias_backward": _exact_bias_backward,
            "token_logprobs": _exact_token_logprobs}[op](case, s)
