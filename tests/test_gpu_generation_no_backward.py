"""Inputs of generation's operators that require a gradient, on the GPU: a backward pass raises,
whichever input it is of and wherever the outputs lie, instead of leaving a gradient out."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def raises(t):
    with pytest.raises(RuntimeError, match="no backward pass"):
        t.float().sum().backward(retain_graph=True)


def cache_of(mz):
    both = torch.zeros(3, 2, 16, 2, 64, device="cuda")
    return both, mz.PagedCache(both[:, 0], both[:, 1], torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3))


def test_frequencies(mz):
    """Learned ones."""
    both, cache = cache_of(mz)
    qkv = torch.randn(5, 6, 64, device="cuda")
    freqs = torch.rand(32, device="cuda", requires_grad=True)
    docs = cache.documents([5], [5])
    out = mz.cache_append(qkv[:, 2:4], qkv[:, 4:], cache, docs, q=qkv[:, :2], freqs=freqs)
    for t in (out, cache.k):
        raises(t)
    both2, cache2 = cache_of(mz)
    with torch.no_grad():
        same = mz.cache_append(qkv[:, 2:4], qkv[:, 4:], cache2, docs, q=qkv[:, :2], freqs=freqs)
    assert torch.equal(same, out) and torch.equal(both, both2) and not same.requires_grad and not both2.requires_grad


def test_scales(mz):
    w = mz.nf4_quantize(torch.randn(10, 64, device="cuda"))
    x = torch.randn(4, 64, device="cuda")
    want = mz.nf4_linear(x, w)
    w.absmax.requires_grad_(True)
    got = mz.nf4_linear(x, w)
    assert torch.equal(got, want)
    raises(got)


@pytest.mark.parametrize("paged", [True, False])
def test_outputs_in_a_wider_array_with_their_lse(mz, paged):
    q = torch.randn(5, 4, 64, device="cuda", requires_grad=True)
    room = torch.zeros(5, 6, 64, device="cuda")
    both, cache = cache_of(mz)
    kv = torch.randn(5, 4, 64, device="cuda")
    docs = cache.documents([5], [5])
    mz.cache_append(kv[:, :2], kv[:, 2:], cache, docs)
    if paged:
        out, lse = mz.paged_attention(q, cache, docs, out=room[:, 1:5], return_lse=True)
        want = mz.paged_attention(q.detach(), cache, docs)
    else:
        out, lse = mz.attention(q, kv[:, :2], kv[:, 2:], docs, out=room[:, 1:5], return_lse=True)
        want = mz.attention(q.detach(), kv[:, :2], kv[:, 2:], docs)
    assert torch.equal(out, want)
    for t in (out, lse, room):
        raises(t)
