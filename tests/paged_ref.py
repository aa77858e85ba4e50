"""Plain references of a paged cache, in 64 bits or more on the CPU: turning by
positions, where tokens go, and attention by visible keys alone. Shares nothing
with the kernels."""
import math

import numpy as np
import torch


def turned(x, positions, freqs, interleaved):
    """x [tokens, heads, dim] turned by positions * freqs (in 80 bits, so that far
    positions keep their angle), and |x_a| + |x_b| of each element's pair, what
    errors of sine and cosine are relative to."""
    x = x.detach().cpu().double().numpy()
    out, size = x.copy(), np.zeros_like(x)
    if freqs is None or len(freqs) == 0:
        return torch.from_numpy(out), torch.from_numpy(size)
    half = len(freqs)
    a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    angle = np.asarray(positions, dtype=np.longdouble)[:, None] * freqs.cpu().double().numpy().astype(np.longdouble)
    c, s = np.cos(angle)[:, None].astype(np.float64), np.sin(angle)[:, None].astype(np.float64)
    out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return torch.from_numpy(out), torch.from_numpy(size)


def turned_bound(want, size, positions, freqs, dtype):
    """How far a turned value may be off. The angle: formed in fp64 (three
    roundings), brought to fp32 as a part of half a turn (2^-24 of at most pi); its
    sine and cosine: 4 steps; a product and a fused one, and the result's rounding."""
    u = 2.0 ** -24
    far = 0.0
    if freqs is not None and len(freqs):
        far = float(np.abs(np.asarray(positions, dtype=np.float64)).max(initial=0.0) * float(freqs.abs().max()))
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else u
    return (math.pi * u + 4 * u + 2 * u + 3 * 2.0 ** -53 * far) * size + rounding * want.abs()


def row(pages, rows, first, j):
    """(page, row of the page) of key j of the document whose list starts at `first`."""
    return int(pages[first + j // rows]), j % rows


def gathered(cache, pages, rows, first, n):
    """The first n keys (or values) of a document, [n, kv_heads, dim]."""
    at = [row(pages, rows, first, j) for j in range(n)]
    return torch.stack([cache[p, r] for p, r in at]) if at else cache.new_zeros((0, *cache.shape[2:]))


def attention(q, k_cache, v_cache, pages, table, causal=True, scale=None, softcap=0.0, slopes=None, follows=None):
    """table = [(q_first, q_len, first entry, k_len, prefix)]; follows: for trees, of
    each query token the set of its document's new tokens that it sees. Returns (out,
    lse, weight) as attention_ref.attention does."""
    q = q.detach().cpu().double()
    kc, vc = (t.detach().cpu().double() for t in (k_cache, v_cache))
    pages, rows = pages.cpu().flatten().tolist(), k_cache.shape[1]
    heads, dim, group = q.shape[1], q.shape[2], q.shape[1] // kc.shape[2]
    scale = 1.0 / math.sqrt(dim) if scale is None else scale
    out, weight = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    for q0, nq, first, nk, prefix in table:
        k, v = gathered(kc, pages, rows, first, nk), gathered(vc, pages, rows, first, nk)
        for i in range(nq):
            pos = i + nk - nq
            if follows is not None:
                seen = [j for j in range(nk) if j < nk - nq or j < prefix or j - (nk - nq) in follows[q0 + i]]
            else:
                seen = list(range(max(pos + 1, prefix, 0) if causal else nk))
            if not seen:
                continue
            for h in range(heads):
                s = scale * (k[seen, h // group] @ q[q0 + i, h])
                if softcap:
                    s = softcap * torch.tanh(s / softcap)
                if slopes is not None:
                    s = s - float(slopes[h]) * (pos - torch.tensor(seen)).abs().double()
                p = torch.softmax(s, 0)
                out[q0 + i, h] = p @ v[seen, h // group]
                weight[q0 + i, h] = p @ v[seen, h // group].abs()
                lse[q0 + i, h] = torch.logsumexp(s, 0)
    return out, lse, weight
