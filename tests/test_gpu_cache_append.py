"""Appending to a paged cache on the GPU, through the binding, against a plain
reference (paged_ref.py): where tokens go, what they are turned by, and what is
left alone. The bars come from the arithmetic (paged_ref.turned_bound)."""
import numpy as np
import pytest
import torch

import paged_ref

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def frequencies(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float().cuda() if rot else None


class Case:
    """New tokens of documents of these lengths, and a cache whose pages are in no order."""

    def __init__(self, mz, q_lens, k_lens, heads=4, kv_heads=2, dim=64, rows=16, dtype="bf16", seed=0, layout="plain"):
        g = torch.Generator().manual_seed(seed + 13 * sum(q_lens) + dim)
        dt = DTYPES[dtype]
        self.mz, self.q_lens, self.k_lens, self.rows, self.dtype = mz, q_lens, k_lens, rows, dt
        tokens, d = sum(q_lens), dim
        qkv = torch.randn(tokens, heads + 2 * kv_heads, d, generator=g).to(dt).cuda()
        self.q, self.k, self.v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        counts = [(n + rows - 1) // rows for n in k_lens]
        self.first = [int(x) for x in np.cumsum([0, *counts])[:-1]]
        n_pages = sum(counts) + 3
        self.pages = torch.randperm(n_pages, generator=g)[:sum(counts)].int()
        shape = (n_pages, rows, kv_heads, d)
        if layout == "plain":
            kc, vc = (torch.randn(*shape, generator=g).to(dt).cuda() for _ in range(2))
        elif layout == "fused":  # a page's keys, then its values
            both = torch.randn(n_pages, 2, rows, kv_heads, d, generator=g).to(dt).cuda()
            kc, vc = both[:, 0], both[:, 1]
        else:  # heads before rows
            kc, vc = (torch.randn(n_pages, kv_heads, rows, d, generator=g).to(dt).cuda().transpose(1, 2) for _ in range(2))
        self.cache = mz.PagedCache(kc, vc, self.pages.cuda())
        self.docs = mz.Documents.of(q_lens, k_lens, k_first=self.first)
        self.places = [n - m + i for m, n in zip(q_lens, k_lens) for i in range(m)]

    def check(self, rot, interleaved=False, positions=None, with_q=True, out=None, q=None):
        freqs = frequencies(rot)
        pos = self.places if positions is None else positions
        k0, v0 = self.cache.k.clone().cpu(), self.cache.v.clone().cpu()
        q = self.q if q is None else q
        want_q, size_q = paged_ref.turned(q, pos, freqs, interleaved)
        want_k, size_k = paged_ref.turned(self.k, pos, freqs, interleaved)
        v = self.v.cpu()
        bound_q = paged_ref.turned_bound(want_q, size_q, pos, freqs, self.dtype)
        bound_k = paged_ref.turned_bound(want_k, size_k, pos, freqs, self.dtype)
        got = self.mz.cache_append(self.k, self.v, self.cache, self.docs, q=q if with_q else None, freqs=freqs,
                                   positions=None if positions is None else torch.tensor(positions, device="cuda"),
                                   interleaved=interleaved, out=out)
        if with_q:
            assert got.dtype == self.dtype and got.shape == q.shape
            assert bool(((got.cpu().double() - want_q).abs() <= bound_q).all())
        else:
            assert got is None
        kc, vc = self.cache.k.cpu(), self.cache.v.cpu()
        token = 0
        for m, n, first in zip(self.q_lens, self.k_lens, self.first):
            for i in range(m):
                place = n - m + i
                if place >= 0:
                    at = paged_ref.row(self.pages, self.rows, first, place)
                    assert bool(((kc[at].double() - want_k[token]).abs() <= bound_k[token]).all()), (token, place)
                    assert torch.equal(vc[at], v[token])
                    k0[at], v0[at] = kc[at], vc[at]
                token += 1
        assert torch.equal(kc, k0) and torch.equal(vc, v0)  # the rest is as it was
        return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 64), (128, 128), (40, 40), (40, 20), (40, 10), (40, 2), (8, 8),
                                     (80, 80), (80, 48), (64, 6), (64, 0), (120, 118)])
def test_sizes_of_heads(mz, dim, rot, interleaved, dtype):
    Case(mz, [1, 5, 40], [30, 5, 45], dim=dim, dtype=dtype).check(rot, interleaved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [8, 16, 64, 256])
@pytest.mark.parametrize("q_lens,k_lens", [([1], [1]), ([1] * 5, [1, 8, 9, 64, 65]), ([0, 3, 0], [4, 3, 0]),
                                           ([17, 200], [17, 333]), ([70], [70])])
def test_documents_and_pages(mz, q_lens, k_lens, rows, dtype):
    Case(mz, q_lens, k_lens, rows=rows, dtype=dtype).check(64)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (12, 12), (32, 8), (3, 1), (7, 5), (40, 40)])
@pytest.mark.parametrize("tokens", [1, 9])
def test_heads(mz, heads, kv_heads, tokens):
    Case(mz, [tokens, tokens], [tokens, 50], heads=heads, kv_heads=kv_heads).check(64)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["fused", "heads"])
def test_layouts_of_the_cache(mz, layout, dtype):
    Case(mz, [3, 20], [33, 20], layout=layout, dtype=dtype).check(64)


def test_many_tokens(mz):
    Case(mz, [700, 1, 900], [900, 77, 900], heads=8, kv_heads=4, dim=128).check(128)


def test_without_queries(mz):
    Case(mz, [4, 9], [4, 40]).check(64, with_q=False)


@pytest.mark.parametrize("interleaved", [False, True])
def test_queries_turned_in_place(mz, interleaved):
    """They and the keys are parts of one array."""
    c = Case(mz, [4, 30], [20, 40])
    before = c.k.clone()
    q = c.q.clone()
    c2 = Case(mz, [4, 30], [20, 40])
    want = c2.check(64, interleaved)
    got = mz.cache_append(c.k, c.v, c.cache, c.docs, q=c.q, freqs=frequencies(64), interleaved=interleaved, out=c.q)
    assert got is c.q and torch.equal(c.q, want) and not torch.equal(c.q, q)
    assert torch.equal(c.k, before) and torch.equal(c.cache.k, c2.cache.k)


@pytest.mark.parametrize("dtype", DTYPES)
def test_given_positions(mz, dtype):
    """Of a tree's tokens; far, negative and past 32 bits."""
    c = Case(mz, [4, 6], [40, 6], dtype=dtype)
    c.check(64, positions=[36, 37, 37, 38, 0, -5, 2 ** 31 - 1, -2 ** 31, 1000003, 7])
    c.check(64, positions=[2 ** 33 + 1] * 10)


def test_places_before_the_first_key_store_nothing(mz):
    """More queries than keys: the first ones stand before the document."""
    Case(mz, [5, 4], [2, 0]).check(64)


def test_entries_outside_the_cache_store_nothing(mz):
    c = Case(mz, [2, 2], [20, 30])
    pages = c.pages.clone()
    pages[1], pages[3] = -1, c.cache.n_pages
    k0, v0 = c.cache.k.clone(), c.cache.v.clone()
    cache = mz.PagedCache(c.cache.k, c.cache.v, pages.cuda())
    got = mz.cache_append(c.k, c.v, cache, c.docs, q=c.q, freqs=frequencies(64))
    want, size = paged_ref.turned(c.q, c.places, frequencies(64), False)
    assert bool(((got.cpu().double() - want).abs()
                 <= paged_ref.turned_bound(want, size, c.places, frequencies(64), c.dtype)).all())
    assert torch.equal(cache.k, k0) and torch.equal(cache.v, v0)


def test_tables_outside_the_arrays_are_cut(mz):
    c = Case(mz, [8], [8])
    k0 = c.cache.k.clone()
    for r in ([-5, 4, 0, 4, 0], [100, 4, 0, 4, 0], [0, 1 << 40, 0, 1 << 40, 0], [0, 4, 1 << 40, 4, 0], [0, 4, -7, -4, 0],
              [6, 100, 0, 100, 0]):
        table = torch.tensor([r], dtype=torch.int64, device="cuda")
        mz.cache_append(c.k, c.v, c.cache, mz.Documents(table, 8, 8), q=c.q, freqs=frequencies(64))
    torch.cuda.synchronize()
    outside = [p for p in range(c.cache.n_pages) if p not in c.pages.tolist()]
    assert torch.equal(c.cache.k[outside], k0[outside])


def test_tokens_of_no_document(mz):
    c = Case(mz, [3, 4], [3, 4])
    docs = mz.Documents.of([3], [3], k_first=[0])
    got = mz.cache_append(c.k, c.v, c.cache, docs, q=c.q, freqs=frequencies(64))
    assert bool((got[3:] == 0).all()) and not bool((got[:3] == 0).all())
    out = torch.full_like(got, 5.0)
    mz.cache_append(c.k, c.v, c.cache, docs, q=c.q, freqs=frequencies(64), out=out)
    assert bool((out[3:] == 5).all()) and torch.equal(out[:3], got[:3])


def test_queries_past_max_q_are_left_out(mz):
    c = Case(mz, [6], [6])
    docs = mz.Documents(c.docs.table, 4, 6)
    out = torch.full(c.q.shape, 5.0, dtype=c.dtype, device="cuda")
    v0 = c.cache.v.clone()
    mz.cache_append(c.k, c.v, c.cache, docs, q=c.q, freqs=frequencies(64), out=out)
    page = int(c.pages[0])
    assert bool((out[4:] == 5).all()) and torch.equal(c.cache.v[page, :4], c.v[:4])
    assert torch.equal(c.cache.v[page, 4:], v0[page, 4:])


def test_values_that_are_not_finite_stay_in_their_pairs(mz):
    c = Case(mz, [2], [2])
    k = c.k.clone().contiguous()
    k[0, 0, 3], k[1, 1, 40] = float("nan"), float("inf")
    mz.cache_append(k, c.v, c.cache, c.docs, freqs=frequencies(64))
    page = int(c.pages[0])
    bad = ~torch.isfinite(c.cache.k[page, :2].float())
    where = {tuple(x) for x in bad.nonzero().tolist()}
    assert where <= {(0, 0, 3), (0, 0, 35), (1, 1, 8), (1, 1, 40)} and (0, 0, 3) in where and len(where) >= 3


def test_empty_calls(mz):
    c = Case(mz, [2], [2])
    k0 = c.cache.k.clone()
    for docs in (mz.Documents.of([], []), mz.Documents.of([0], [0])):
        got = mz.cache_append(c.k, c.v, c.cache, docs, q=c.q, freqs=frequencies(64))
        assert bool((got == 0).all())
    assert torch.equal(c.cache.k, k0)
    none = mz.cache_append(c.k[:0], c.v[:0], c.cache, mz.Documents.of([0], [0]), q=c.q[:0], freqs=frequencies(64))
    assert none.shape == (0, 4, 64)


def test_another_stream_and_a_graph(mz):
    c = Case(mz, [1, 1, 1], [20, 33, 5])
    want = c.check(64)
    wk = c.cache.k.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.cache.k.zero_()
    side.wait_stream(torch.cuda.current_stream())
    got = mz.cache_append(c.k, c.v, c.cache, c.docs, q=c.q, freqs=frequencies(64), stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    # captured: replays read the table, the inputs and the list as they are then
    freqs, out = frequencies(64), torch.empty(c.q.shape, dtype=c.dtype, device="cuda")
    q, k, v = c.q.clone(), c.k.clone(), c.v.clone()
    table = c.docs.table.clone()
    docs = mz.Documents(table, 1, 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mz.cache_append(k, v, c.cache, docs, q=q, freqs=freqs, out=out)
    for step in range(3):
        table[:, 3] = c.docs.table[:, 3] - step
        k.copy_(c.k * (step + 1))
        q.copy_(c.q * (step + 1))
        c.cache.k.copy_(wk)
        graph.replay()
        replayed, rk = out.clone(), c.cache.k.clone()
        torch.cuda.synchronize()
        c.cache.k.copy_(wk)
        eager = mz.cache_append(k, v, c.cache, docs, q=q, freqs=freqs)
        assert torch.equal(replayed, eager) and torch.equal(rk, c.cache.k)


def test_no_backward(mz):
    c = Case(mz, [2], [2])
    k = c.k.clone().requires_grad_(True)
    q = c.q.clone().requires_grad_(True)
    got = mz.cache_append(k, c.v, c.cache, c.docs, q=q, freqs=frequencies(64))
    for t in (got, c.cache.k, c.cache.v):
        with pytest.raises(RuntimeError, match="no backward pass"):
            t.float().sum().backward(retain_graph=True)
    with torch.no_grad():
        assert not mz.cache_append(k, c.v, Case(mz, [2], [2]).cache, c.docs, q=q).requires_grad


def test_more_workgroups_than_a_row_of_a_grid(mz):
    """A padded batch: 2^16 documents of up to 512 tokens, nearly all of them without any."""
    heads, dim, rows, tokens = 64, 128, 16, 512
    docs = 1 << 16
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(tokens, heads, dim, generator=g).cuda() for _ in range(3))
    table = torch.zeros(docs, 5, dtype=torch.int64)
    table[0] = torch.tensor([0, 5, 0, 5, 0])
    table[-1] = torch.tensor([5, 507, 1, 507, 0])
    pages = torch.randperm(33, generator=g).int()
    cache = mz.PagedCache(torch.zeros(33, rows, heads, dim, device="cuda"), torch.zeros(33, rows, heads, dim, device="cuda"),
                          pages.cuda())
    out = mz.cache_append(k, v, cache, mz.Documents(table.cuda(), tokens, tokens), q=q)
    assert torch.equal(out, q)
    for new, where in ((k, cache.k), (v, cache.v)):
        flat = where[pages.long().cuda()].reshape(33 * rows, heads, dim)
        assert torch.equal(flat[:5], new[:5]) and torch.equal(flat[rows:rows + 507], new[5:])
        assert not flat[5:rows].any() and not flat[rows + 507:].any()
