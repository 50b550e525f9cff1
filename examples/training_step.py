"""A training step as a rank takes it, on one GPU: what the library does at each message.

Two data-parallel ranks share one model (both run here, one after the other): a projection whose two tensor-parallel halves are
summed up by an all-reduce of bf16 messages, a join with the residual stream with norms around it, and a squared loss.  Per step

    forward    each tensor-parallel half's output is compressed, reduced and decompressed (zc_compress_half, zc_reduce_decompress),
               joins the residual stream and is normed (zt_residual_norm)
    backward   zt_residual_norm_backward, whose sums over rows go into the fp32 gradient bucket beside the projection's gradient
    exchange   the bucket is compressed, summed over the ranks and decompressed (zc_compress, zc_reduce_compressed, zc_decompress)
    update     the norm over all gradients (zt_sum_squares, of each rank's half of the bucket), then each rank's shard is
               updated with the clipped gradients (zt_adamw) and leaves its parameters in bf16 for the lossless all-gather (zl_compress16,
               zl_decompress16)

    python examples/training_step.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2409_02423_amd import zc, zt  # noqa: E402

RANKS, TOKENS, INPUTS, HIDDEN = 2, 512, 128, 500
GRADIENT_RATE = zc.zc_rate_for_class(zc.ZC_DP_GRADIENT)
ACTIVATION_RATE = zc.zc_rate_for_class(zc.ZC_TP_ACTIVATION)
FORM = dict(kind=zt.ZT_RMS, post=True, residual_scale=1.0)
ADAM = dict(lr=2e-2, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.01)
MAX_NORM = 0.5


class Model:
    """The parameters as the ranks hold them: bf16 for the products, fp32 with its moments in one shard a rank."""

    def __init__(self, generator):
        sizes = (INPUTS * HIDDEN, HIDDEN, HIDDEN, HIDDEN)
        start = torch.cat([torch.randn(sizes[0], generator=generator, device="cuda") / INPUTS ** 0.5, torch.ones(2 * HIDDEN, device="cuda"),
                           torch.full((HIDDEN,), 0.5, device="cuda")])
        self.shards = [[t, torch.zeros_like(t), torch.zeros_like(t)] for t in (s.clone() for s in start.chunk(RANKS))]
        self.half = start.bfloat16()
        self.weight, self.pre, self.post, self.gate = self.half.split(sizes)

    def forms(self):
        return dict(pre_weight=self.pre, post_weight=self.post, d_gate=self.gate, **FORM)


def projection(inputs, weight):
    """inputs @ weight, its two halves along the inputs on two tensor-parallel ranks and summed up by their all-reduce."""
    w = weight.view(INPUTS, HIDDEN)
    messages = [zc.zc_compress_half(a @ b, ACTIVATION_RATE) for a, b in zip(inputs.chunk(2, 1), w.chunk(2, 0))]
    return zc.zc_reduce_decompress(messages, None, TOKENS * HIDDEN, ACTIVATION_RATE).view(TOKENS, HIDDEN).bfloat16()


def gradients(model, inputs, residual, target):
    """One rank's loss and its gradient bucket."""
    block = projection(inputs, model.weight)
    stats = torch.empty((TOKENS, 4), device="cuda")
    y, h = zt.zt_residual_norm(residual, block, d_stats=stats, **model.forms())
    difference = h.float() - target
    dh = (difference / TOKENS).bfloat16()
    d = zt.zt_residual_norm_backward(None, dh, y, block, stats, **model.forms())
    d_weight = inputs.t().float() @ d["b"].float()
    bucket = torch.cat([d_weight.reshape(-1), d["pre_weight"], d["post_weight"], d["gate"]])
    return float(0.5 * difference.square().sum() / TOKENS), bucket


def step(model, batches, number):
    losses, buckets = zip(*(gradients(model, *batch) for batch in batches))
    n = buckets[0].numel()
    total = zc.zc_reduce_compressed([zc.zc_compress(b, GRADIENT_RATE) for b in buckets], n, GRADIENT_RATE)
    reduced = zc.zc_decompress(total, n, GRADIENT_RATE)
    shards = reduced.chunk(RANKS)
    # each rank squares its shard, and an all-reduce adds the slots up
    slots = sum(zt.zt_sum_squares([g]) for g in shards)
    messages = []
    for rank, (grad, (param, m, v)) in enumerate(zip(shards, model.shards)):
        half = torch.empty(grad.numel(), dtype=torch.bfloat16, device="cuda")
        norm = zt.zt_adamw(grad, param, m, v, step=number, d_half=half, d_slots=slots, scale=1.0 / RANKS, max_norm=MAX_NORM, **ADAM)
        messages.append((zl(half), half.numel()))
    model.half.copy_(torch.cat([zc.zl_decompress16(stream, count) for stream, count in messages]))
    return sum(losses) / RANKS, float(norm)


def zl(half):
    stream = zc.zl_compress16(half)
    return stream[:zc.zl_stream_bytes(stream)]


def main(steps=30):
    g = torch.Generator(device="cuda").manual_seed(1)

    def draw(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    truth = draw(INPUTS, HIDDEN) / INPUTS ** 0.5
    batches = []
    for _ in range(RANKS):
        inputs, residual = draw(TOKENS, INPUTS).bfloat16(), draw(TOKENS, HIDDEN).bfloat16()
        target = residual.float() + inputs.float() @ truth
        batches.append((inputs, residual, target / target.square().mean(1, keepdim=True).sqrt()))
    model = Model(g)
    history = []
    for number in range(1, steps + 1):
        history.append(step(model, batches, number))
        print("step %3d  loss %8.4f  gradient norm %.4f" % (number, *history[-1]), flush=True)
    return history


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 30)
