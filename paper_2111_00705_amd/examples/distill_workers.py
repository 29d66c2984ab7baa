"""A small language model distilled from a larger one's top logits by n workers through the compressed optimiser.

The student is one transformer block with a learned relative position bias (in place of position embeddings).  Everything that a
worker's microbatch contributes is computed for all workers at once, and the gradient of every parameter goes per worker into
grads[n, d], which CompAms.step compresses and averages: norm gains and shifts, the bias table and the loss by the library's
operators, matrix parameters by batched products over the workers.  The teacher (random weights) is asked once per batch for its
best tokens, as a recorded teacher would be.

With --eight-bits the student runs and keeps its activations in 8 bits: root-mean-square norms whose results leave in 8 bits, products of 8-bit
integers, and weight gradients formed from the 8-bit rows that the products read.  Gradients go straight through the roundings.

    python -m paper_2111_00705_amd.examples.distill_workers [--iterations 60] [--workers 8] [--eight-bits]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.dirname(os.path.abspath(__file__)))))

VOCAB, WIDTH, HEADS, LENGTH, BUCKETS, TOP, TEMPERATURE = 2000, 128, 4, 48, 16, 16, 2.0


class Layout:
    """Where each parameter stands in the flat model."""

    def __init__(self, shapes):
        self.at, self.shape, self.d = {}, shapes, 0
        for name, shape in shapes.items():
            size = 1
            for s in shape:
                size *= s
            self.at[name] = (self.d, self.d + size)
            self.d += size

    def view(self, flat, name):
        """The parameter in theta [d], or its gradients per worker in grads [n, d]."""
        lo, hi = self.at[name]
        return flat[lo:hi].view(self.shape[name]) if flat.dim() == 1 else flat[:, lo:hi].unflatten(1, self.shape[name])


def layout():
    return Layout({"embed": (VOCAB, WIDTH), "g1": (WIDTH,), "b1": (WIDTH,), "qkv": (WIDTH, 3 * WIDTH), "bias": (BUCKETS, HEADS),
                   "out": (WIDTH, WIDTH), "g2": (WIDTH,), "b2": (WIDTH,), "head": (WIDTH, VOCAB)})


def distill_iteration(P, lay, theta, grads, tokens, lengths, idx, val, bounds):
    """Forward and backward pass of all workers; returns the mean loss of each (a tensor of n).  tokens [n, batch, length]."""
    import torch
    n, batch, length = tokens.shape
    rows, dim = n * batch * length, WIDTH // HEADS
    p = {name: lay.view(theta, name) for name in lay.shape}
    g = {name: lay.view(grads, name) for name in lay.shape}
    per_worker = lambda t: t.view(n, batch * length, -1)

    x0 = p["embed"][tokens.view(-1)]                                                   # [rows, WIDTH]
    y1, mean1, rstd1 = P.layer_norm(x0, p["g1"], p["b1"])
    qkv = (y1 @ p["qkv"]).view(n * batch, length, 3, HEADS, dim).permute(2, 0, 3, 1, 4).contiguous()
    q, k, v = qkv[0], qkv[1], qkv[2]
    kt = k.transpose(-1, -2).contiguous()
    probs = P.rel_bias_softmax(torch.matmul(q, kt), p["bias"], bounds, scale=dim ** -0.5, causal=True, key_lengths=lengths)
    mixed = torch.matmul(probs, v).transpose(1, 2).reshape(rows, WIDTH)
    x1 = x0 + mixed @ p["out"]
    y2, mean2, rstd2 = P.layer_norm(x1, p["g2"], p["b2"])
    logits = y2 @ p["head"]

    weight = torch.full((rows,), 1.0 / (batch * length), device=theta.device)           # each worker's loss is its mean
    loss, dlogits = P.distill_grad(logits, idx, val, weight, temperature=TEMPERATURE, out=logits)

    g["head"].copy_(torch.bmm(per_worker(y2).transpose(1, 2).contiguous(), per_worker(dlogits)))
    dy2 = dlogits @ p["head"].t().contiguous()
    dx1 = P.layer_norm_backward(dy2, x1, mean2, rstd2, p["g2"], g["g2"], g["b2"], out=dy2)
    g["out"].copy_(torch.bmm(per_worker(mixed).transpose(1, 2).contiguous(), per_worker(dx1)))
    dmixed = (dx1 @ p["out"].t().contiguous()).view(n * batch, length, HEADS, dim).transpose(1, 2).contiguous()
    dprobs = torch.matmul(dmixed, v.transpose(-1, -2).contiguous())
    dv = torch.matmul(probs.transpose(-1, -2).contiguous(), dmixed)
    dscores = P.rel_bias_softmax_backward(dprobs, probs, bounds, g["bias"], scale=dim ** -0.5, causal=True, key_lengths=lengths, out=dprobs)
    dq, dk = torch.matmul(dscores, k), torch.matmul(dscores.transpose(-1, -2).contiguous(), q)
    dqkv = torch.stack([dq, dk, dv]).permute(1, 3, 0, 2, 4).reshape(rows, 3 * WIDTH)
    g["qkv"].copy_(torch.bmm(per_worker(y1).transpose(1, 2).contiguous(), per_worker(dqkv)))
    dy1 = dqkv @ p["qkv"].t().contiguous()
    dx0 = dx1 + P.layer_norm_backward(dy1, x0, mean1, rstd1, p["g1"], g["g1"], g["b1"], out=dy1)
    g["embed"].zero_()
    for w in range(n):
        g["embed"][w].index_add_(0, tokens[w].view(-1), per_worker(dx0)[w])
    return loss.view(n, -1).mean(1)


def distill_iteration_eight_bits(P, lay, theta, grads, tokens, lengths, idx, val, bounds):
    """The same for a student with root-mean-square norms (b1 and b2 are not used) whose products take 8 bits.  What is kept for the backward
    pass of a product is the 8-bit rows that it read."""
    import torch
    n, batch, length = tokens.shape
    rows, dim = n * batch * length, WIDTH // HEADS
    p = {name: lay.view(theta, name) for name in lay.shape}
    g = {name: lay.view(grads, name) for name in lay.shape}
    f32 = theta.dtype
    weights = {name: P.quantize_rows(p[name].t().contiguous()) for name in ("qkv", "out", "head")}        # [outs, cols], a scale for each channel

    def product(kept, name):
        return P.linear_q8(*kept, *weights[name], dtype=f32)

    def product_backward(dy, kept, name):
        P.linear_weight_grad(dy, *kept, g[name].transpose(1, 2), binary=True)
        return dy @ P.restore_rows(*weights[name], f32)

    x0 = p["embed"][tokens.view(-1)]                                                   # [rows, WIDTH]
    *kept1, _, rstd1 = P.rms_norm_q8(x0, p["g1"], binary=True)
    qkv = product(kept1, "qkv").view(n * batch, length, 3, HEADS, dim).permute(2, 0, 3, 1, 4).contiguous()
    q, k, v = qkv[0], qkv[1], qkv[2]
    probs = P.rel_bias_softmax(torch.matmul(q, k.transpose(-1, -2).contiguous()), p["bias"], bounds, scale=dim ** -0.5, causal=True, key_lengths=lengths)
    mixed = P.quantize_rows(torch.matmul(probs, v).transpose(1, 2).reshape(rows, WIDTH), binary=True)
    *kept2, x1, rstd2 = P.rms_norm_q8(product(mixed, "out"), p["g2"], x0, binary=True)
    logits = product(kept2, "head")

    weight = torch.full((rows,), 1.0 / (batch * length), device=theta.device)           # each worker's loss is its mean
    loss, dlogits = P.distill_grad(logits, idx, val, weight, temperature=TEMPERATURE, out=logits)

    dx1 = P.rms_norm_backward(product_backward(dlogits, kept2, "head"), x1, rstd2, p["g2"], g["g2"])
    dmixed = product_backward(dx1, mixed, "out").view(n * batch, length, HEADS, dim).transpose(1, 2).contiguous()
    dprobs = torch.matmul(dmixed, v.transpose(-1, -2).contiguous())
    dv = torch.matmul(probs.transpose(-1, -2).contiguous(), dmixed)
    dscores = P.rel_bias_softmax_backward(dprobs, probs, bounds, g["bias"], scale=dim ** -0.5, causal=True, key_lengths=lengths, out=dprobs)
    dq, dk = torch.matmul(dscores, k), torch.matmul(dscores.transpose(-1, -2).contiguous(), q)
    dqkv = torch.stack([dq, dk, dv]).permute(1, 3, 0, 2, 4).reshape(rows, 3 * WIDTH)
    dx0 = P.rms_norm_backward(product_backward(dqkv, kept1, "qkv"), x0, rstd1, p["g1"], g["g1"], dresidual=dx1)
    g["b1"].zero_()
    g["b2"].zero_()
    g["embed"].zero_()
    for w in range(n):
        g["embed"][w].index_add_(0, tokens[w].view(-1), dx0.view(n, batch * length, -1)[w])
    return loss.view(n, -1).mean(1)


def run(iterations=60, n=8, batch=4, seed=0, report=None, eight_bits=False):
    """Distils; returns (mean loss before each iteration, bits per step and worker, the same without compression)."""
    import torch

    import paper_2111_00705_amd as P
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lay = layout()
    theta = torch.randn(lay.d, device="cuda", generator=gen) * 0.05
    for name in ("g1", "g2"):
        lay.view(theta, name).fill_(1.0)
    for name in ("b1", "b2", "bias"):
        lay.view(theta, name).zero_()
    teacher = torch.randn(VOCAB, VOCAB, device="cuda", generator=gen) * 2.0              # logits after each token
    tokens = torch.randint(0, VOCAB, (n, batch, LENGTH), device="cuda", generator=gen)
    lengths = torch.randint(LENGTH // 2, LENGTH + 1, (n * batch,), device="cuda", generator=gen).to(torch.int32)
    _, _, idx, val = P.token_logprobs(teacher[tokens.view(-1)], None, TOP)
    bounds = P.rel_bias_bounds(BUCKETS, LENGTH, causal=True)
    grads = torch.zeros(n, lay.d, device="cuda")
    h = P.CompAms(lay.d, n, P.TOPK, lay.d // 50, 0.9, 0.999, 1e-8, 3e-3)
    h.set_theta(theta)
    losses = []
    iteration = distill_iteration_eight_bits if eight_bits else distill_iteration
    for t in range(iterations):
        loss = iteration(P, lay, theta, grads, tokens, lengths, idx, val, bounds)
        losses.append(float(loss.mean()))
        if report and t % 10 == 0:
            report(f"{t:9d} {losses[-1]:12.4f}")
        h.step(grads)
        h.get_theta(out=theta)
    bits = sum(h.message_bits())
    h.destroy()
    return losses, bits, 64 * lay.d


def main() -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--iterations", type=int, default=60)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--eight-bits", action="store_true")
    args = ap.parse_args()
    import torch
    assert torch.cuda.is_available(), "this example needs a GPU"
    print(f"{args.workers} workers, vocabulary {VOCAB}, the teacher's {TOP} best tokens\niteration    mean loss")
    losses, bits, dense = run(args.iterations, args.workers, report=print, eight_bits=args.eight_bits)
    print(f"{args.iterations:9d} {losses[-1]:12.4f}   bits per step and worker (up + down) {bits}, uncompressed {dense}")
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
