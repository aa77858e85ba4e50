"""Equal inputs give equal bits in the operators of generation, again and on another stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def again(f):
    first = [t.clone() for t in f(None)]
    side = torch.cuda.Stream()
    for i in range(6):
        if i == 3:
            side.wait_stream(torch.cuda.current_stream())
        got = f(side if i >= 3 else None)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("q_lens,k_lens,tree", [([1] * 6, [20, 4000, 700, 1, 9000, 300], False),  # keys split, joined
                                                ([61, 61], [3000, 5000], True), ([200, 1, 333], [2000, 50, 333], False),
                                                ([100] * 40, [100 + 37 * i for i in range(40)], False)])  # longest first
def test_attention_and_append(mz, q_lens, k_lens, tree, dtype):
    heads, kv_heads, dim, rows = 8, 2, 128, 16
    g = torch.Generator("cuda").manual_seed(sum(k_lens))
    entries = (max(k_lens) + rows - 1) // rows
    pages = torch.randperm(len(q_lens) * entries, generator=g, device="cuda").int().view(len(q_lens), entries)
    k, v = (torch.randn(len(q_lens) * entries, rows, kv_heads, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
    cache = mz.PagedCache(k, v, pages)
    docs = cache.documents(q_lens, k_lens)
    qkv = torch.randn(sum(q_lens), heads + 2 * kv_heads, dim, generator=g, device="cuda").to(dtype)
    freqs = torch.rand(64, generator=g, device="cuda")
    mask = mz.tree_mask([[max(-1, i - 1 - i % 3) for i in range(n)] for n in q_lens])[0] if tree else None

    def step(stream):
        q = mz.cache_append(qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], cache, docs, q=qkv[:, :heads],
                            freqs=freqs, stream=stream)
        out, lse = mz.paged_attention(q, cache, docs, tree=mask, return_lse=True, stream=stream)
        return q, out, lse, cache.k, cache.v

    again(step)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (24, 1000, 8192), (40, 333, 5000), (300, 303, 2000), (1100, 333, 2000)])
def test_products(mz, m, n, k, dtype):
    g = torch.Generator("cuda").manual_seed(m)
    w = mz.nf4_quantize(torch.randn(n, k, generator=g, device="cuda"))
    x = torch.randn(m, k, generator=g, device="cuda").to(dtype)
    again(lambda stream: (mz.nf4_linear(x, w, stream=stream),))
