"""Appends of more than 64 MB on the GPU, whose kernels store around the caches: turned by
either order of pairs, in both types, by vectors of every length, against turns in 64 bits
there. The bars are those of paged_ref.turned_bound."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ROWS = 16


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def turned(x, places, freqs, interleaved):
    """As the formula has it, in 64 bits, and how far each value may be off."""
    x, out = x.double(), x.double()
    half = freqs.numel()
    a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    t = (places.double()[:, None] * freqs.double())[:, None]
    size = torch.zeros_like(x)
    out[..., a], out[..., b] = (x[..., a] * t.cos() - x[..., b] * t.sin(), x[..., a] * t.sin() + x[..., b] * t.cos())
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 48), (64, 24), (128, 20), (64, 6), (128, 0)])
def test_large_appends(mz, dim, rot, interleaved, dtype):
    heads, kv_heads, dt = 24, 8, DTYPES[dtype]
    q_lens, k_lens = [4000, 1, 2101, 0], [4000, 700, 3500, 5]
    tokens, capacity = sum(q_lens), 4000 // ROWS
    assert len(q_lens) * max(q_lens) * (heads + 2 * kv_heads) * dim * dt.itemsize > 64 << 20
    g = torch.Generator("cuda").manual_seed(dim + rot)
    qkv = torch.randn(tokens, heads + 2 * kv_heads, dim, generator=g, device="cuda").to(dt)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    pages = torch.randperm(4 * capacity + 3, generator=g, device="cuda")[:4 * capacity].int().view(4, capacity)
    both = torch.randn(2, 4 * capacity + 3, ROWS, kv_heads, dim, generator=g, device="cuda").to(dt)
    before = both.clone()
    cache = mz.PagedCache(both[0], both[1], pages)
    freqs = (10000.0 ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float().cuda()
    got = mz.cache_append(k, v, cache, cache.documents(q_lens, k_lens), q=q, freqs=freqs, interleaved=interleaved)
    places = torch.cat([torch.arange(n - m, n) for m, n in zip(q_lens, k_lens)]).cuda()
    documents = torch.repeat_interleave(torch.arange(4), torch.tensor(q_lens)).cuda()
    rows = pages[documents, places // ROWS].long() * ROWS + places % ROWS
    u, rounding = 2.0 ** -24, 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    flat = before.view(2, -1, kv_heads, dim)
    for x, out in ((q, got), (k, cache.k.reshape(-1, kv_heads, dim)[rows])):
        want, size = turned(x, places, freqs, interleaved)
        bar = ((math.pi + 6) * u + 3 * 2.0 ** -53 * 4000) * size + rounding * want.abs()
        assert bool(((out.double() - want).abs() <= bar).all())
    flat[0, rows], flat[1, rows] = cache.k.reshape(-1, kv_heads, dim)[rows], v
    assert torch.equal(both, before)  # the values as they were, and nothing else was written
