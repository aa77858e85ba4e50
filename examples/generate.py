"""Tuning by generated answers, on 4-bit weights, end to end on one GPU.

What is scored here has no derivative: the share of an answer's words that are
wrong. The engine perturbs the weights in their 4-bit storage, products read that
storage as it is (nothing is written out or quantized again), and answers are
generated over a paged cache: the prompts in one pass, then a word of each at a time.
With --draft every pass checks a tree of guesses instead and keeps the longest
right path, which gives the same words in fewer passes.

    python examples/generate.py [--steps 30] [--samples 8] [--draft]

The task is synthetic: the words of an answer are to be from the first half of the
vocabulary.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2306_10015_amd import mezo  # noqa: E402

PAGE = 16


class Decoder:
    """A decoder whose layers (qkv, out, up, down each) and last product are in
    4-bit storage, in one list in registration order (= tensor_id)."""

    def __init__(self, vocab=64, width=128, heads=4, kv_heads=2, ffn=256, layers=2, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.width, self.heads, self.kv_heads, self.dim, self.layers = width, heads, kv_heads, width // heads, layers
        shapes = []
        for _ in range(layers):
            shapes += [((heads + 2 * kv_heads) * self.dim, width), (width, width), (ffn, width), (width, ffn)]
        shapes.append((vocab, width))
        self.weights = [mezo.nf4_quantize(torch.empty(s, device="cuda").normal_(0, s[1] ** -0.5, generator=g))
                        for s in shapes]
        self.words = torch.empty(vocab, width, device="cuda").normal_(0, 1, generator=g).to(dtype)
        exponent = torch.arange(0, self.dim, 2, device="cuda", dtype=torch.float64) / self.dim
        self.freqs = (10000.0 ** -exponent).float()

    def caches(self, documents, capacity):
        """One paged cache a layer for `documents` of up to `capacity` words, with one list of pages."""
        entries = (capacity + PAGE - 1) // PAGE
        pages = torch.randperm(documents * entries, device="cuda").int().view(documents, entries)
        return [mezo.PagedCache.empty(documents * entries, PAGE, self.kv_heads, self.dim, pages, self.words.dtype)
                for _ in range(self.layers)]

    def logits(self, words, caches, docs, tree=None, positions=None):
        """The next word's logits after each of the documents' new words, which go into the caches."""
        norm = torch.nn.functional.rms_norm
        x = self.words[words]
        h, hk, d = self.heads, self.kv_heads, self.dim
        for i, cache in enumerate(caches):
            qkv_w, out_w, up_w, down_w = self.weights[4 * i:4 * i + 4]
            qkv = mezo.nf4_linear(norm(x, (self.width,)), qkv_w).view(-1, h + 2 * hk, d)
            q = mezo.cache_append(qkv[:, h:h + hk], qkv[:, h + hk:], cache, docs, q=qkv[:, :h], freqs=self.freqs,
                                  positions=positions)
            a = mezo.paged_attention(q, cache, docs, tree=tree)
            x = x + mezo.nf4_linear(a.flatten(1), out_w)
            x = x + mezo.nf4_linear(torch.relu(mezo.nf4_linear(norm(x, (self.width,)), up_w)), down_w)
        return mezo.nf4_linear(norm(x, (self.width,)), self.weights[-1], torch.float32)


def greedy(model, prompts, count):
    """`count` words after each prompt (a list of lists), one pass a word."""
    lens = [len(p) for p in prompts]
    caches = model.caches(len(prompts), max(lens) + count)
    last = torch.tensor([sum(lens[:i + 1]) - 1 for i in range(len(lens))], device="cuda")
    words = torch.tensor([w for p in prompts for w in p], device="cuda")
    new = model.logits(words, caches, caches[0].documents(lens, lens))[last].argmax(1)
    out = [new]
    for step in range(1, count):
        docs = caches[0].documents([1] * len(lens), [n + step for n in lens])
        new = model.logits(new, caches, docs).argmax(1)
        out.append(new)
    return torch.stack(out, 1)


def drafted(model, prompts, count, guesses):
    """The same words, a tree a pass: `guesses(document, words so far)` gives (words, parents)
    of a tree that continues them. Returns (words, passes)."""
    lens = [len(p) for p in prompts]
    room = max(lens) + count + 32
    caches = model.caches(len(prompts), room)
    words = torch.tensor([w for p in prompts for w in p], device="cuda")
    logits = model.logits(words, caches, caches[0].documents(lens, lens)).argmax(1).tolist()
    answers = [[logits[sum(lens[:i + 1]) - 1]] for i in range(len(lens))]
    passes = 1
    while min(map(len, answers)) < count:
        # each document: its last word, whose keys are not in the cache yet, and the tree below it
        trees, parents = [], []
        for i, a in enumerate(answers):
            w, p = guesses(i, a) if len(a) < count else ([], [])
            trees.append([a[-1], *w[:31]])
            parents.append([-1, *(x + 1 for x in p[:31])])
        mask, depth = mezo.tree_mask(parents)
        n_new = [len(t) for t in trees]
        kept = [lens[i] + len(answers[i]) - 1 for i in range(len(lens))]
        positions = depth + torch.tensor([k for k, n in zip(kept, n_new) for _ in range(n)], device="cuda")
        docs = caches[0].documents(n_new, [k + n for k, n in zip(kept, n_new)])
        nxt = model.logits(torch.tensor([w for t in trees for w in t], device="cuda"), caches, docs, mask,
                           positions).argmax(1).tolist()
        passes += 1
        at, paths = 0, []
        for i, (tree, up) in enumerate(zip(trees, parents)):
            node, path = 0, [0]
            while len(answers[i]) < count:
                word = nxt[at + node]
                answers[i].append(word)
                below = [t for t in range(len(tree)) if up[t] == node and t > node and tree[t] == word]
                if not below:
                    break
                node = below[0]
                path.append(node)
            paths.append(path)
            at += len(tree)
        keep(caches, kept, paths)
    return torch.tensor(answers, device="cuda"), passes


def keep(caches, kept, paths):
    """Move the rows of each document's right path behind its old ones (a row never moves up)."""
    entries = caches[0].pages.shape[1]
    for cache in caches:
        pages = cache.pages.cpu()
        for i, path in enumerate(paths):
            for to, t in enumerate(path):
                if to != t:
                    (a, b), (c, d) = (divmod(kept[i] + x, PAGE) for x in (t, to))
                    a, c = int(pages[i, a]), int(pages[i, c])
                    cache.k[c, d], cache.v[c, d] = cache.k[a, b], cache.v[a, b]
        assert entries * PAGE >= max(kept) + max(map(len, paths))


def batch(vocab, count, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    lens = torch.randint(3, 20, (count,), generator=g).tolist()
    return [torch.randint(0, vocab, (n,), generator=g).tolist() for n in lens]


def guess_repeats(i, answer):
    """A model that is not tuned yet repeats itself: its last word again, or its last two."""
    a, b = answer[-2:] if len(answer) > 1 else (answer[0], answer[0])
    return [b, b, b, a, b, a], [-1, 0, 1, -1, 3, 4]


def train(steps=30, samples=8, eps=2e-2, eta=1e-2, count=64, answer=4, draft=False, seed=0, report=None):
    """Run `steps` iterations; the mean share of wrong words at each one's start."""
    vocab = 64
    model = Decoder(vocab=vocab, seed=seed)
    backup = [mezo.NF4Tensor(w.codes.clone(), w.absmax.clone(), w.numel()) for w in model.weights]
    theta, probe = mezo.ParamSet(backup), mezo.ParamSet(model.weights)
    codec = mezo.codec(mezo.LINEAR, scale=0.25)
    history = []
    for step in range(steps):
        prompts = batch(vocab, count, seed * 100_003 + step)

        def wrong():
            got = drafted(model, prompts, answer, guess_repeats)[0] if draft else greedy(model, prompts, answer)
            return (got >= vocab // 2).float().mean()

        seeds, grads = [(1, step, j) for j in range(samples)], []
        for s in seeds:
            probe.perturb_from(theta, s, +eps)
            plus = wrong()
            probe.perturb_from(theta, s, -eps)
            minus = wrong()
            grads.append((plus - minus) / (2 * eps))
            if s is seeds[0]:
                history.append((plus + minus) / 2)
        q = mezo.quantize_projgrad(torch.stack(grads).cpu().numpy(), codec)
        theta.update_multi(seeds, q, mezo.step_lr(eta, samples), codec)
        if report and step % report == 0:
            print(f"step {step}: {100 * float(history[-1]):.1f}% of the words wrong", flush=True)
    return [float(x) for x in history]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--samples", type=int, default=8)
    ap.add_argument("--draft", action="store_true")
    args = ap.parse_args()
    train(args.steps, args.samples, draft=args.draft, report=max(1, args.steps // 10))


if __name__ == "__main__":
    main()
