"""Attention over a paged cache on the GPU, through the binding, against a plain
reference in 64 bits (paged_ref.py): pages that end inside tiles, trees of drafted
tokens, and whatever lies in the cache that a query does not see. The bars come
from the arithmetic (attention_ref.bounds)."""
import math

import numpy as np
import pytest
import torch

import attention_ref
import paged_ref

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


class Case:
    def __init__(self, mz, q_lens, k_lens, heads=4, kv_heads=2, dim=64, rows=16, dtype="bf16", prefix=None, seed=0,
                 layout="plain", stale=float("nan")):
        g = torch.Generator().manual_seed(seed + 13 * sum(k_lens) + dim)
        dt = DTYPES[dtype]
        self.mz, self.rows = mz, rows
        self.q = (torch.randn(sum(q_lens), heads, dim, generator=g) * 1.5).to(dt).cuda()
        counts = [(n + rows - 1) // rows for n in k_lens]
        self.first = [int(x) for x in np.cumsum([0, *counts])[:-1]]
        n_pages = sum(counts) + 2
        self.pages = torch.randperm(n_pages, generator=g)[:sum(counts)].int()
        k = (torch.randn(n_pages, rows, kv_heads, dim, generator=g) * 1.5).to(dt)
        v = torch.randn(n_pages, rows, kv_heads, dim, generator=g).to(dt)
        # rows of no document: never used
        used = torch.zeros(n_pages, rows, dtype=torch.bool)
        for n, first in zip(k_lens, self.first):
            for j in range(n):
                used[paged_ref.row(self.pages, rows, first, j)] = True
        k[~used], v[~used] = stale, stale
        self.clean = torch.nan_to_num(k, 0.0, 0.0, 0.0), torch.nan_to_num(v, 0.0, 0.0, 0.0)
        if layout == "fused":
            both = torch.stack((k, v), 1).cuda()
            k, v = both[:, 0], both[:, 1]
        elif layout == "heads":
            k, v = (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (k, v))
        else:
            k, v = k.cuda(), v.cuda()
        self.cache = mz.PagedCache(k, v, self.pages.cuda())
        q_first = [int(x) for x in np.cumsum([0, *q_lens])[:-1]]
        self.table = list(zip(q_first, q_lens, self.first, k_lens, prefix or [0] * len(q_lens)))
        self.docs = mz.Documents.of(q_lens, k_lens, prefix, k_first=self.first)

    def check(self, parents=None, **kw):
        """Against the reference; parents: of the new tokens' trees."""
        tree = follows = None
        if parents is not None:
            tree = self.mz.tree_mask(parents)[0]
            follows = []
            for t in parents:
                own = []
                for i, p in enumerate(t):
                    own.append((own[p] if p >= 0 else set()) | {i})
                follows += own
        out, lse = self.mz.paged_attention(self.q, self.cache, self.docs, tree=tree, return_lse=True, **kw)
        return self.compare(out, lse, follows, **kw)

    def compare(self, out, lse, follows=None, **kw):
        q = self.q
        assert out.dtype == q.dtype and out.shape == q.shape and lse.shape == q.shape[:2]
        kw.pop("out", None)
        want, want_lse, weight = paged_ref.attention(q, *self.clean, self.pages, self.table, follows=follows, **kw)
        kw.pop("causal", None)
        ob, lb = attention_ref.bounds(want, want_lse, weight, q.float(), self.clean[0].float(), q.dtype,
                                      max([r[3] for r in self.table], default=0), **kw)
        off = (out.cpu().double() - want).abs()
        assert bool((off <= ob).all()), float((off / ob).max())
        got, empty = lse.cpu().double(), torch.isinf(want_lse)
        assert bool((got[empty] == -math.inf).all())
        assert bool(((got - want_lse).abs()[~empty] <= lb[~empty]).all())
        return out, lse


def chain(n):
    return list(range(-1, n - 1))


def random_tree(n, seed):
    r = np.random.default_rng(seed)
    return [int(r.integers(max(-1, t - 6), t)) if t else -1 for t in range(n)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [8, 40, 64, 80, 128])
@pytest.mark.parametrize("rows", [8, 16, 64, 128])
def test_single_tokens(mz, rows, dim, dtype):
    k_lens = [1, 7, 8, 31, 32, 33, 64, 65, 200]
    Case(mz, [1] * len(k_lens), k_lens, dim=dim, rows=rows, dtype=dtype).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [8, 32, 256])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (3, 3, 64), (8, 1, 40)])
@pytest.mark.parametrize("nq", [2, 5, 17, 70])
def test_new_tokens(mz, nq, heads, kv_heads, dim, rows, dtype):
    Case(mz, [nq] * 3, [nq, 129, 95], heads, kv_heads, dim, rows, dtype).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_whole_documents_and_prefixes(mz, causal, dtype):
    lens = [1, 37, 0, 64, 150]
    Case(mz, lens, lens, dtype=dtype, prefix=[0, 5, 0, 64, 33]).check(causal=causal)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("softcap,bias,scale", [(30.0, False, None), (0.0, True, None), (5.0, True, 0.3),
                                                (300.0, False, None), (0.0, False, -0.2)])
def test_score_functions(mz, softcap, bias, scale, dim, dtype):
    slopes = torch.tensor([0.5, 0.03, 0.0, -0.01], device="cuda") if bias else None
    for q_lens, k_lens in (([70, 60], [70, 150]), ([1, 2], [80, 61])):
        Case(mz, q_lens, k_lens, dim=dim, dtype=dtype, prefix=[10, 0]).check(softcap=softcap, slopes=slopes, scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["fused", "heads"])
def test_layouts_of_the_cache(mz, layout, dtype):
    Case(mz, [1, 40], [90, 77], layout=layout, dtype=dtype).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (4, 4, 64), (2, 1, 40)])
@pytest.mark.parametrize("nq", [1, 2, 7, 31, 61, 64, 65, 130])
def test_trees(mz, nq, heads, kv_heads, dim, dtype):
    c = Case(mz, [nq, nq, nq], [nq, nq + 45, nq + 96], heads, kv_heads, dim, 16, dtype)
    c.check([random_tree(nq, 1), chain(nq), [-1] * nq])


@pytest.mark.parametrize("dtype", DTYPES)
def test_trees_of_several_sizes_with_capped_scores(mz, dtype):
    n = [3, 0, 70, 1, 33]
    c = Case(mz, n, [40, 20, 100, 1, 33], 4, 1, 64, 8, dtype)
    parents = [random_tree(x, 5 + x) for x in n]
    c.check(parents, softcap=20.0)
    c.check(parents, scale=0.4)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_chain_is_causal(mz, dtype):
    for nq, nk in ((5, 70), (80, 300), (64, 64)):
        c = Case(mz, [nq], [nk], dtype=dtype)
        plain = mz.paged_attention(c.q, c.cache, c.docs, return_lse=True)
        tree = mz.paged_attention(c.q, c.cache, c.docs, tree=mz.tree_mask([chain(nq)])[0], return_lse=True)
        assert torch.equal(plain[0], tree[0]) and torch.equal(plain[1], tree[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq", [3, 40])
@pytest.mark.parametrize("nk", [3, 40, 500, 700])
def test_masks_that_leave_nothing(mz, nk, nq, dtype):
    """Rows without a bit, over a context or none; also where the keys are split."""
    nk = max(nk, nq)
    c = Case(mz, [nq], [nk], dtype=dtype)
    mask = mz.tree_mask([chain(nq)])[0]
    mask[1] = 0
    mask[2] = 2  # not itself
    out, lse = mz.paged_attention(c.q, c.cache, c.docs, tree=mask, return_lse=True)
    follows = [set(range(i + 1)) for i in range(nq)]
    follows[1], follows[2] = set(), {1}
    c.compare(out, lse, follows)
    if nk == nq:
        assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_bits_past_the_new_tokens_and_words_that_are_missing(mz, dtype):
    c = Case(mz, [70], [170], dtype=dtype)
    full = mz.tree_mask([random_tree(70, 3)])[0]
    want = mz.paged_attention(c.q, c.cache, c.docs, tree=full, return_lse=True)
    more = torch.cat((full, torch.full((70, 1), -1, dtype=torch.int64, device="cuda")), 1)
    more[:, 1] |= -1 << 6  # bits of tokens 70 .. 127, of which there are none
    got = mz.paged_attention(c.q, c.cache, c.docs, tree=more, return_lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # one word: tokens from 64 on are seen by nobody
    short = full[:, :1].contiguous()
    out, lse = mz.paged_attention(c.q, c.cache, c.docs, tree=short, return_lse=True)
    follows = [{b for b in range(64) if int(x) >> b & 1} for x in short[:, 0].tolist()]
    c.compare(out, lse, follows)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("nq,nk", [(4, 60), (40, 60), (4, 700), (40, 700)])
def test_hidden_keys_that_are_not_finite(mz, nq, nk, bad, dtype):
    """A drafted token's values reach those alone that follow it."""
    c = Case(mz, [nq], [nk], dtype=dtype)
    parents = [-1, 0, 0] + [1] * (nq - 3)  # token 2 has no descendant
    page, row = paged_ref.row(c.pages, c.rows, 0, nk - nq + 2)
    for t in (c.cache.k, c.cache.v):
        t[page, row] = bad
    tree = mz.tree_mask([parents])[0]
    out, lse = mz.paged_attention(c.q, c.cache, c.docs, tree=tree, return_lse=True)
    rest = [i for i in range(nq) if i != 2]
    assert not bool(torch.isfinite(out[2].float()).any())
    c.clean[0][page, row], c.clean[1][page, row] = 0, 0
    follows = []
    for i, p in enumerate(parents):
        follows.append((follows[p] if p >= 0 else set()) | {i})
    want, want_lse, weight = paged_ref.attention(c.q, *c.clean, c.pages, c.table, follows=follows)
    ob, lb = attention_ref.bounds(want, want_lse, weight, c.q.float(), c.clean[0].float(), c.q.dtype, nk)
    assert bool(((out.cpu().double() - want).abs() <= ob)[rest].all())
    assert bool(((lse.cpu().double() - want_lse).abs() <= lb)[rest].all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("q_lens,k_lens,heads,kv_heads,dim", [
    ([1, 1], [3000, 40], 8, 2, 128), ([1], [5000], 4, 4, 64), ([64], [2100], 4, 1, 64), ([200], [1500], 2, 2, 128)])
def test_split_keys(mz, q_lens, k_lens, heads, kv_heads, dim, dtype):
    c = Case(mz, q_lens, k_lens, heads, kv_heads, dim, 32, dtype)
    c.check()
    c.check([random_tree(n, 9) for n in q_lens])


def test_contiguous_pages_give_what_contiguous_keys_give(mz):
    """The same keys in pages in order: the same sums in the same order."""
    for dtype in DTYPES.values():
        g = torch.Generator().manual_seed(3)
        for nq, nk in ((1, 333), (50, 333), (1, 4000)):
            q = torch.randn(nq, 8, 128, generator=g).to(dtype).cuda()
            k, v = (torch.randn((nk + 15) // 16 * 16, 2, 128, generator=g).to(dtype).cuda() for _ in range(2))
            want = mz.attention(q, k[:nk], v[:nk], mz.Documents.of([nq], [nk]), return_lse=True)
            pages = torch.arange(len(k) // 16, dtype=torch.int32, device="cuda")[None]
            cache = mz.PagedCache(k.view(-1, 16, 2, 128), v.view(-1, 16, 2, 128), pages)
            got = mz.paged_attention(q, cache, cache.documents([nq], [nk]), return_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_shared_pages(mz):
    """Two documents with the same first pages."""
    c = Case(mz, [1, 1], [64, 40])
    pages = torch.tensor([[0, 1, 2, 3], [0, 1, 4, 4]], dtype=torch.int32, device="cuda")
    k = torch.randn(5, 16, 2, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(0)).bfloat16()
    v = torch.randn(5, 16, 2, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    cache = mz.PagedCache(k, v, pages)
    c.cache, c.pages, c.clean = cache, pages.flatten().cpu(), (k.cpu(), v.cpu())
    c.docs = cache.documents([1, 1], [64, 40])
    c.table = [(0, 1, 0, 64, 0), (1, 1, 4, 40, 0)]
    c.check()


def test_entries_outside_the_cache_and_tables_outside_the_list(mz):
    """What comes out is unspecified but for the rows of other documents; nothing outside is read."""
    c = Case(mz, [1, 1], [40, 40], stale=0.0)
    want = mz.paged_attention(c.q, c.cache, c.docs)
    pages = c.pages.clone()
    pages[4], pages[5] = -3, 1 << 30
    cache = mz.PagedCache(c.cache.k, c.cache.v, pages.cuda())
    out = mz.paged_attention(c.q, cache, c.docs)
    assert torch.equal(out[0], want[0]) and bool(torch.isfinite(out.float()).all())
    last = pages.clone()
    last[4:] = c.cache.n_pages - 1
    as_last = mz.paged_attention(c.q, mz.PagedCache(c.cache.k, c.cache.v, torch.cat((pages[:4], last[4:])).cuda()), c.docs)
    assert as_last.shape == out.shape
    # a list that is shorter than the keys it is said to have: cut to it
    table = torch.tensor([[0, 1, 0, 10 ** 9, 0], [1, 1, 4, 10 ** 9, 0]], dtype=torch.int64, device="cuda")
    cut = mz.paged_attention(c.q, c.cache, mz.Documents(table, 1, 96))
    exact = torch.tensor([[0, 1, 0, 96, 0], [1, 1, 4, 32, 0]], dtype=torch.int64, device="cuda")
    assert torch.equal(cut, mz.paged_attention(c.q, c.cache, mz.Documents(exact, 1, 96)))
    for r in ([-1, 1, 99, 5, 0], [5, 1, 0, 5, 0], [0, 1, -4, -5, -6]):
        mz.paged_attention(c.q, c.cache, mz.Documents(torch.tensor([r, r], device="cuda"), 1, 40))
    torch.cuda.synchronize()


def test_empty_calls(mz):
    c = Case(mz, [2], [20])
    out, lse = mz.paged_attention(c.q, c.cache, mz.Documents.of([], []), return_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    docs = mz.Documents.of([2], [0])
    out, lse = mz.paged_attention(c.q, c.cache, docs, return_lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    assert mz.paged_attention(c.q[:0], c.cache, mz.Documents.of([0], [20])).shape == (0, 4, 64)
    none = mz.PagedCache(c.cache.k[:0], c.cache.v[:0], c.pages.cuda())
    out = mz.paged_attention(c.q, none, c.docs)
    assert bool((out == 0).all())


def test_long_cache_past_32_bits(mz):
    """Pages more than 4 GiB apart."""
    rows, dim = 256, 128
    n_pages = (5 << 30) // (rows * dim * 2)
    k = torch.zeros(n_pages, rows, 1, dim, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator("cuda").manual_seed(0)
    far = [n_pages - 1, 0, n_pages - 2]
    for p in far:
        k[p].normal_(generator=g)
        v[p].normal_(generator=g)
    small = mz.PagedCache(k[far].contiguous(), v[far].contiguous(), torch.arange(3, dtype=torch.int32, device="cuda")[None])
    big = mz.PagedCache(k, v, torch.tensor([far], dtype=torch.int32, device="cuda"))
    for nq in (1, 100):
        q = torch.empty(nq, 1, dim, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        docs = small.documents([nq], [700])
        assert torch.equal(mz.paged_attention(q, small, docs), mz.paged_attention(q, big, docs))
    kn, vn = k[0, :2].clone(), v[0, :2].clone()
    mz.cache_append(kn, vn, big, mz.Documents.of([2], [702], k_first=[0]))
    assert torch.equal(k[n_pages - 2, 700 - 512:702 - 512], kn)


def test_outputs_given_and_tokens_of_no_document(mz):
    c = Case(mz, [3, 4], [30, 40])
    want, want_lse = mz.paged_attention(c.q, c.cache, c.docs, return_lse=True)
    wide = torch.full((7, 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    got = mz.paged_attention(c.q, c.cache, c.docs, out=wide[:, :, 64:])
    assert torch.equal(got, want) and bool((wide[:, :, :64] == 5).all())
    docs = mz.Documents.of([4], [40], q_first=[3], k_first=[c.first[1]])
    docs.covered = 0
    out, lse = mz.paged_attention(c.q, c.cache, docs, return_lse=True)
    assert torch.equal(out[3:], want[3:]) and bool((out[:3] == 0).all()) and bool((lse[:3] == -math.inf).all())


def test_another_stream_and_graphs(mz):
    """Two captured calls with workspaces, replayed in turn with changed lists and tables."""
    c = Case(mz, [1, 1], [3000, 600], 8, 2, 128, 32, stale=0.0)
    want = mz.paged_attention(c.q, c.cache, c.docs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mz.paged_attention(c.q, c.cache, c.docs, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    table, pages, q = c.docs.table.clone(), c.cache.pages.clone(), c.q.clone()
    cache = mz.PagedCache(c.cache.k, c.cache.v, pages)
    docs = mz.Documents(table, 1, 3000)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        out = torch.empty_like(q)
        with torch.cuda.graph(g):
            mz.paged_attention(q, cache, docs, out=out)
        graphs.append(g)
        outs.append(out)
    for step in range(4):
        table[:, 3] = c.docs.table[:, 3] - 37 * step
        pages.copy_(c.cache.pages.roll(step))
        q.copy_(c.q * (1 + step))
        graphs[step % 2].replay()
        got = outs[step % 2].clone()
        torch.cuda.synchronize()
        assert torch.equal(got, mz.paged_attention(q, cache, docs))
        graphs[1 - step % 2].replay()
        assert torch.equal(outs[0], outs[1])


def test_no_backward(mz):
    c = Case(mz, [1], [20])
    q = c.q.clone().requires_grad_(True)
    out, lse = mz.paged_attention(q, c.cache, c.docs, return_lse=True)
    for t in (out, lse):
        with pytest.raises(RuntimeError, match="no backward pass"):
            t.float().sum().backward(retain_graph=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("docs", [2, 63, 64, 65])
def test_order_of_documents(mz, docs, dtype):
    """Of up to 64 documents the longest goes first: equal lengths, none at all, and queries of
    no document's order; a table that says more keys than there are."""
    r = np.random.default_rng(docs)
    k_lens = [int(n) for n in r.choice([0, 1, 40, 40, 129, 250], docs)]
    q_lens = [int(n) for n in r.choice([0, 1, 33, 70, 150], docs)]
    q_lens[-1], k_lens[-1] = 150, 250
    c = Case(mz, q_lens, k_lens, heads=3, kv_heads=3, dtype=dtype)
    out, lse = c.check()
    c.docs.table[:-1, 3][c.docs.table[:-1, 1] == 0] = 1 << 62
    again, lse_again = mz.paged_attention(c.q, c.cache, c.docs, return_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse_again)
