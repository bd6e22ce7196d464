"""Prune the output layer of a language model to DARB form and retrain what it keeps.

The model's last layer reads hidden states h, normalises them, and gives each word a logit:
Z = W LN(h).  W is pruned by magnitude, its row densities set the block sizes, and the layer
from there on is W's retained values in DARB form (paper section 3).  Retraining (section 4.1)
moves those values and the layer norm's weight and bias down the gradient of the words'
negative log probability, with the pattern held fixed:

    forward    LN -> DARB product -> log probabilities
    backward   logits -> DARB product (values and input) -> LN (weight and bias)
    update     AdamW on values, weight and bias, in one launch

Synthetic data: W is drawn, and every word is drawn from the distribution that the dense layer
gives its hidden state, so that the dense layer is the best one and pruning costs perplexity.

    python examples/retrain_output_layer.py [--steps 300] [--values f16] [--state-bits 8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1911_08020_amd as darb  # noqa: E402
import workloads  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16}


class OutputLayer:
    """Layer norm and a DARB product, with what a training step of them needs."""

    def __init__(self, plan, values, offsets, hidden: int, state_bits: int = 32, lr: float = 1e-3):
        self.plan, self.values, self.offsets = plan, values, offsets
        self.index = plan.transpose(offsets)                  # the pattern by columns, once
        self.weight = torch.ones(hidden, device="cuda")
        self.bias = torch.zeros(hidden, device="cuda")
        # 16-bit values step through fp32 copies; the layer norm's two vectors do not decay
        self.opt = darb.AdamW([values, self.weight, self.bias], lr=lr, masters=True,
                              state_bits=state_bits, weight_decay=[0.01, 0.0, 0.0])

    def logits(self, h):
        x, mean, rstd = darb.layer_norm(h, self.weight, self.bias)
        return self.plan.spmm(self.values, self.offsets, x), (x, mean, rstd)

    def evaluate(self, h, words, top: int = 5):
        """(perplexity, share of words among the `top` most likely)."""
        r = darb.token_logprobs(self.logits(h)[0], words, top=top)
        hit = (r.top_index == words[:, None]).any(1)
        return math.exp(-r.logprob.mean().item()), hit.float().mean().item()

    def gradients(self, h, words):
        """(mean log probability, [d values, d weight, d bias]) of minus that mean."""
        z, (x, mean, rstd) = self.logits(h)
        r = darb.token_logprobs(z, words)
        g = torch.full_like(r.logprob, -1.0 / words.numel())
        dz = darb.token_logprobs_grad(z, words, r.lse, g, out=z)
        dvalues, dx = self.plan.spmm_grad(self.index, self.values, x, dz)
        _, dweight, dbias = darb.layer_norm_grad(dx, h, mean, rstd, self.weight, need_x=False)
        return r.logprob.mean(), [dvalues, dweight, dbias]

    def step(self, h, words, lr=None):
        logprob, grads = self.gradients(h, words)
        self.opt.step(grads, lr=lr)
        return logprob


def make_data(W, tokens: int, seed: int):
    """Hidden states [hidden, tokens] and a word for each, from the dense layer W."""
    rng = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(W.shape[1], tokens, device="cuda", generator=rng) * 2.0 + 0.5
    z = W @ torch.nn.functional.layer_norm(h.t(), W.shape[1:]).t()
    words = torch.multinomial(torch.softmax(z.t(), 1), 1, generator=rng)[:, 0]
    return h, words, z


def prune(W, keep: float, b_min: int, b_max: int, dtype):
    """W [M, N] -> (plan, values, offsets), on the device."""
    k = int(math.floor(keep * W.numel() + 0.5))
    counts = darb.prune_counts(W, k)
    plan = darb.Plan.from_device_counts(W.shape[1], counts, k, darb.ROUND_FLOOR, b_min, b_max)
    values, offsets = plan.encode(W)
    return plan, values.to(dtype), offsets


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--words", type=int, default=10000)
    p.add_argument("--hidden", type=int, default=1500)
    p.add_argument("--keep", type=float, default=0.065, help="share of W that pruning keeps")
    p.add_argument("--batch", type=int, default=700, help="tokens of a step (35 steps of a batch of 20)")
    p.add_argument("--batches", type=int, default=300, help="different batches to train on")
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--lr", type=float, default=2e-3)
    p.add_argument("--values", choices=sorted(TYPES), default="f32")
    p.add_argument("--state-bits", type=int, choices=(32, 8), default=32)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args(argv)

    m = workloads.make_matrix(a.words, a.hidden, dist="laplace", keep=a.keep, seed=a.seed)
    # logits of standard deviation 3 under unit hidden states, whatever the sizes
    W = torch.from_numpy(m.W).cuda()
    W *= 3.0 / W.pow(2).sum(1).mean().sqrt()
    train = [make_data(W, a.batch, a.seed + 1 + i)[:2] for i in range(a.batches)]
    h, words, z = make_data(W, a.batch, a.seed + 1 + a.batches)        # held out
    dense = math.exp(-darb.token_logprobs(z, words).logprob.mean().item())

    plan, values, offsets = prune(W, a.keep, 4, 64, TYPES[a.values])
    layer = OutputLayer(plan, values, offsets, a.hidden, a.state_bits, a.lr)
    pruned, hits = layer.evaluate(h, words)
    print(f"{a.words} x {a.hidden}, {plan.nnz} weights kept ({100 * plan.nnz / W.numel():.1f} %)")
    print(f"perplexity, held out: dense {dense:.1f}, pruned {pruned:.1f} (top 5: {100 * hits:.1f} %)")
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for i in range(a.steps):
        lr = a.lr * 0.5 * (1.0 + math.cos(math.pi * i / a.steps))
        logprob = layer.step(*train[i % a.batches], lr=lr)
        if (i + 1) % 100 == 0:
            print(f"step {i + 1}: training perplexity {math.exp(-logprob.item()):.1f}", flush=True)
    end.record()
    torch.cuda.synchronize()
    after, hits = layer.evaluate(h, words)
    print(f"perplexity, held out: retrained {after:.1f} (top 5: {100 * hits:.1f} %); "
          f"{1e3 * start.elapsed_time(end) / max(a.steps, 1):.0f} us a step")
    return dense, pruned, after


if __name__ == "__main__":
    main()
