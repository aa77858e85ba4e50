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
