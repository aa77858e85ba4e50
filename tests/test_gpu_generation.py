"""The operators of generation together, as a decoder calls them: prompts, then
single words, then trees of drafted words, each operator's output against its
reference in 64 bits from the very values it was given; and the example."""
import os
import sys

import pytest
import torch

import attention_ref
import paged_ref
from oracle import nf4

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADS, KV, DIM, WIDTH, ROWS = 4, 2, 32, 128, 8


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import generate
    finally:
        sys.path.pop(0)
    return generate


def linear(mz, x, w, n):
    """A product, checked: sums of k products (six parts each of an fp32 one) and the rounding."""
    out = mz.nf4_linear(x, w)
    k = x.shape[1]
    values = torch.from_numpy(nf4.table()).cuda()
    codes = torch.stack((w.codes & 15, w.codes >> 4), 1).flatten()[:n * k].int()
    wv = (values[codes] * w.absmax.repeat_interleave(64)[:n * k]).view(n, k).to(x.dtype).double()
    want, size = x.double() @ wv.t().contiguous(), x.double().abs() @ wv.abs().t().contiguous()
    steps, rounding = (6 * k + 8, 2.0 ** -24) if x.dtype == torch.float32 else (k + 8, 2.0 ** -8)
    assert bool(((out.double() - want).abs() <= steps * 2.0 ** -24 * size + rounding * want.abs()).all())
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_prompts_words_and_trees(mz, dtype):
    g = torch.Generator("cuda").manual_seed(5)
    rows = (HEADS + 2 * KV) * DIM
    w_in = mz.nf4_quantize(torch.empty(rows, WIDTH, device="cuda").normal_(0, 0.1, generator=g))
    w_out = mz.nf4_quantize(torch.empty(WIDTH, HEADS * DIM, device="cuda").normal_(0, 0.1, generator=g))
    freqs = (10000.0 ** (-torch.arange(0, DIM, 2).double() / DIM)).float().cuda()
    pages = torch.randperm(3 * 12, generator=torch.Generator().manual_seed(1)).int().view(3, 12)
    cache = mz.PagedCache.empty(36, ROWS, KV, DIM, pages.cuda(), dtype)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    lens = [5, 17, 40]
    trees = [[-1, 0, 0, 1], [-1, 0, 1, 2, 3], [-1, -1, 0, 1, 1, 3]]
    for step, q_lens in enumerate((lens, [1, 1, 1], [1, 1, 1], [len(t) for t in trees])):
        k_lens = lens if step == 0 else [a + b for a, b in zip(k_lens, q_lens)]
        docs = cache.documents(q_lens, k_lens)
        mask = positions = follows = None
        places = [n - m + i for m, n in zip(q_lens, k_lens) for i in range(m)]
        if step == 3:
            mask, depth = mz.tree_mask(trees)
            first = [n - m for m, n in zip(q_lens, k_lens) for _ in range(m)]
            positions = depth + torch.tensor(first, device="cuda")
            places = positions.tolist()
            follows = []
            for t in trees:
                own = []
                for i, p in enumerate(t):
                    own.append((own[p] if p >= 0 else set()) | {i})
                follows += own
        x = torch.empty(sum(q_lens), WIDTH, device="cuda").normal_(generator=g).to(dtype)
        qkv = linear(mz, x, w_in, rows).view(-1, HEADS + 2 * KV, DIM)
        q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
        turned = mz.cache_append(k, v, cache, docs, q=q, freqs=freqs, positions=positions)
        for got, given in ((turned, q),):
            want, size = paged_ref.turned(given, places, freqs, False)
            assert bool(((got.cpu().double() - want).abs()
                         <= paged_ref.turned_bound(want, size, places, freqs, dtype)).all())
        want_k, size_k = paged_ref.turned(k, places, freqs, False)
        bound_k = paged_ref.turned_bound(want_k, size_k, places, freqs, dtype)
        kc, vc, token = cache.k.cpu(), cache.v.cpu(), 0
        for d, (m, n) in enumerate(zip(q_lens, k_lens)):
            for i in range(m):
                at = paged_ref.row(pages.flatten(), ROWS, 12 * d, n - m + i)
                assert bool(((kc[at].double() - want_k[token]).abs() <= bound_k[token]).all())
                assert torch.equal(vc[at], v[token].cpu())
                token += 1
        out, lse = mz.paged_attention(turned, cache, docs, tree=mask, return_lse=True)
        table = [(sum(q_lens[:d]), q_lens[d], 12 * d, k_lens[d], 0) for d in range(3)]
        kn, vn = torch.nan_to_num(kc, 0.0), torch.nan_to_num(vc, 0.0)
        want, want_lse, weight = paged_ref.attention(turned, kn, vn, pages, table, follows=follows)
        ob, lb = attention_ref.bounds(want, want_lse, weight, turned.float(), kn.float(), dtype, max(k_lens))
        assert bool(((out.cpu().double() - want).abs() <= ob).all())
        assert bool(((lse.cpu().double() - want_lse).abs() <= lb).all())
        linear(mz, out.flatten(1), w_out, WIDTH)


def test_the_step_in_a_graph(mz):
    """A word's pass captured once and replayed as the documents grow."""
    g = torch.Generator("cuda").manual_seed(5)
    rows = (HEADS + 2 * KV) * DIM
    w_in = mz.nf4_quantize(torch.empty(rows, WIDTH, device="cuda").normal_(0, 0.1, generator=g))
    freqs = (10000.0 ** (-torch.arange(0, DIM, 2).double() / DIM)).float().cuda()
    pages = torch.randperm(2 * 12, device="cuda").int().view(2, 12)
    caches = [mz.PagedCache.empty(24, ROWS, KV, DIM, pages, torch.bfloat16) for _ in range(2)]
    for c in caches:
        c.k.zero_()
        c.v.zero_()
    docs = mz.Documents(caches[0].documents([1, 1], [3, 60]).table, 1, 96)
    x, out = torch.empty(2, WIDTH, dtype=torch.bfloat16, device="cuda"), torch.empty(2, HEADS, DIM, dtype=torch.bfloat16, device="cuda")

    def step(cache, out):
        qkv = mz.nf4_linear(x, w_in).view(-1, HEADS + 2 * KV, DIM)
        q = mz.cache_append(qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:], cache, docs, q=qkv[:, :HEADS], freqs=freqs)
        return mz.paged_attention(q, cache, docs, out=out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], out)
    for i in range(6):
        x.normal_(generator=g)
        docs.table[:, 3] += 1
        graph.replay()
        replayed = out.clone()
        torch.cuda.synchronize()
        want = step(caches[1], None)
        assert torch.equal(replayed, want) and torch.equal(caches[0].k, caches[1].k)


@pytest.mark.parametrize("draft", [False, True])
def test_the_example_runs(example, draft):
    history = example.train(steps=2, samples=2, count=8, draft=draft)
    assert len(history) == 2 and all(0.0 <= h <= 1.0 for h in history)


def test_drafted_words_are_the_greedy_ones(example):
    """In fp32, where no two words come as near as the sums' order moves them."""
    model = example.Decoder(dtype=torch.float32, seed=3)
    prompts = example.batch(64, 12, 7)
    want = example.greedy(model, prompts, 9)
    for guesses in (example.guess_repeats,
                    # every other document is guessed right
                    lambda i, a: (w := want[i, len(a):len(a) + 5].tolist() if i % 2 else [63] * 5, [-1, 0, 1, 2, 3][:len(w)])):
        got, passes = example.drafted(model, prompts, 9, guesses)
        assert torch.equal(got, want) and passes <= 9
