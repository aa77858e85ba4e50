"""Forward-only fine-tuning of a small decoder, end to end on one GPU.

Algorithm 1 with everything in the library: the engine perturbs the weights and
applies the update, and the two forward passes of each sample run on 8-bit
weights quantized after the perturbation, attention over a packed batch of
documents, and the token loss. No gradient is taken and no activation kept.

    python examples/forward_only.py [--steps 200] [--samples 8]

The task is a synthetic classification by prompt: each document's words come
mostly from one of two halves of the vocabulary, and the word after its question
mark names the half. Only that word's loss counts; the prompt is visible both ways
(a prefix).
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2306_10015_amd import mezo  # noqa: E402

MARK, FIRST, SECOND = 0, 1, 2  # the question mark, and the names of the halves


class Decoder:
    """A decoder of `layers` layers, weights in one list in registration order
    (= tensor_id): the embedding, then per layer qkv, out, up, down. Norms have
    no weights; positions enter as a bias by distance."""

    def __init__(self, vocab=64, width=128, heads=4, kv_heads=2, ffn=512, layers=2, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.width, self.heads, self.kv_heads, self.dim = width, heads, kv_heads, width // heads
        rows = (heads + 2 * kv_heads) * self.dim
        shapes = [(vocab, width)]
        for _ in range(layers):
            shapes += [(rows, width), (width, width), (ffn, width), (width, ffn)]
        self.weights = [torch.empty(s, device="cuda").normal_(0, s[1] ** -0.5, generator=g).to(dtype) for s in shapes]
        # 8-bit copies, one buffer each for all forward passes
        self.stored = [mezo.F8Matrix.empty(*s) for s in shapes]
        self.slopes = torch.tensor([2.0 ** -(h + 1) for h in range(heads)], dtype=torch.float32, device="cuda")

    def loss(self, words, targets, docs) -> torch.Tensor:
        """The mean loss of the tokens with a target, at the present weights."""
        for w, q in zip(self.weights, self.stored):
            mezo.f8_quantize(w, out=q)
        norm = torch.nn.functional.rms_norm
        x = self.weights[0][words]
        h, hk, d = self.heads, self.kv_heads, self.dim
        for i in range(1, len(self.stored), 4):
            qkv_w, out_w, up_w, down_w = self.stored[i:i + 4]
            qkv = mezo.f8_linear(norm(x, (self.width,)), qkv_w).view(-1, h + 2 * hk, d)
            a = mezo.attention(qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:], docs, slopes=self.slopes)
            x = x + mezo.f8_linear(a.flatten(1), out_w)
            x = x + mezo.f8_linear(torch.relu(mezo.f8_linear(norm(x, (self.width,)), up_w)), down_w)
        logits = mezo.f8_linear(norm(x, (self.width,)), self.stored[0], torch.float32)
        return mezo.token_loss(logits, targets)[1]


def batch(vocab, count, seed):
    """`count` documents of 3 to 12 words, packed; only the last word has a target."""
    g = torch.Generator()
    g.manual_seed(seed)
    words, targets, lens = [], [], []
    half = (vocab - 3) // 2
    for _ in range(count):
        n, which = int(torch.randint(3, 13, (1,), generator=g)), int(torch.randint(0, 2, (1,), generator=g))
        other = torch.rand(n, generator=g) < 0.1
        doc = 3 + torch.randint(0, half, (n,), generator=g) + half * (other != bool(which)).long()
        words += [*doc.tolist(), MARK]
        targets += [-1] * n + [(FIRST, SECOND)[which]]
        lens.append(n + 1)
    docs = mezo.Documents.of(lens, prefix=lens)
    return torch.tensor(words, device="cuda"), torch.tensor(targets, device="cuda"), docs


def train(steps=200, samples=8, eps=3e-3, eta=1e-3, count=64, seed=0, report=None):
    """Run `steps` iterations and return the loss at each one's start."""
    vocab = 64
    model = Decoder(vocab=vocab, seed=seed)
    backup = [w.clone() for w in model.weights]
    theta = mezo.ParamSet(backup)             # the weights: updated, never perturbed
    probe = mezo.ParamSet(model.weights)      # what the forward passes read
    codec = mezo.codec(mezo.LINEAR, scale=0.25)
    history = []
    for step in range(steps):
        data = batch(vocab, count, seed * 100_003 + step)
        seeds = [(1, step, j) for j in range(samples)]
        grads = []
        for s in seeds:
            probe.perturb_from(theta, s, +eps)
            plus = model.loss(*data)
            probe.perturb_from(theta, s, -eps)
            minus = model.loss(*data)
            grads.append((plus - minus) / (2 * eps))
            if s is seeds[0]:
                history.append((plus + minus) / 2)
        q = mezo.quantize_projgrad(torch.stack(grads).cpu().numpy(), codec)
        theta.update_multi(seeds, q, mezo.step_lr(eta, samples), codec)
        if report and step % report == 0:
            print(f"step {step}: loss {float(history[-1]):.4f}", flush=True)
    return [float(x) for x in history]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--samples", type=int, default=8)
    args = ap.parse_args()
    history = train(args.steps, args.samples, report=max(1, args.steps // 10))
    k = max(1, len(history) // 10)
    print(f"mean loss of the first {k} steps {sum(history[:k]) / k:.4f}, of the last {k} {sum(history[-k:]) / k:.4f}")


if __name__ == "__main__":
    main()
