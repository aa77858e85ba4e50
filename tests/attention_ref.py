"""Plain reference of attention over documents, in 64 bits on the CPU: every
query by its visible keys alone. Shares nothing with the kernels."""
import math

import torch


def attention(q, k, v, rows, causal=True, scale=None, softcap=0.0, slopes=None):
    """q [tokens, heads, dim], k and v [tokens, kv_heads, dim]; rows =
    [(q_first, q_len, k_first, k_len, prefix)]. Returns (out, lse, weight), weight
    = sum_j p_j |v_j| of each element, what roundings of p are relative to."""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    heads, dim, group = q.shape[1], q.shape[2], q.shape[1] // k.shape[1]
    scale = 1.0 / math.sqrt(dim) if scale is None else scale
    out, weight = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    for q0, nq, k0, nk, prefix in rows:
        for i in range(nq):
            pos = i + nk - nq
            n = max(pos + 1, prefix, 0) if causal else nk
            if n == 0:
                continue
            for h in range(heads):
                s = scale * (k[k0:k0 + n, h // group] @ q[q0 + i, h])
                if softcap:
                    s = softcap * torch.tanh(s / softcap)
                if slopes is not None:
                    s = s - float(slopes[h]) * (pos - torch.arange(n)).abs().double()
                p = torch.softmax(s, 0)
                out[q0 + i, h] = p @ v[k0:k0 + n, h // group]
                weight[q0 + i, h] = p @ v[k0:k0 + n, h // group].abs()
                lse[q0 + i, h] = torch.logsumexp(s, 0)
    return out, lse, weight


def bounds(out, lse, weight, q, k, dtype, keys, scale=None, softcap=0.0, slopes=None):
    """How far a kernel's out and lse may be off, element by element: with e the
    error of a score (a sum of dim products and what the score function adds to
    it), p is off by e of itself twice over (numerator and sum) and by its
    rounding, sums of n terms by n u, the result by its rounding."""
    u = 2.0 ** -24
    dim = q.shape[2]
    scale = 1.0 / math.sqrt(dim) if scale is None else abs(scale)
    top = scale * dim * float(q.abs().max()) * float(k.abs().max()) if k.numel() else 0.0  # the largest score
    e = u * (dim + 8) * top
    if softcap:
        e = e + (4 * u if dtype == torch.float32 else 8 * u) * softcap
        top = min(top, softcap)
    if slopes is not None:
        far = float(slopes.abs().max()) * keys
        e = e + 4 * u * far
        top += far
    e = e + 8 * u * top + 4 * u  # scaling, the difference from the reference, exp2
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    out_bound = (2 * e + 2 * keys * u + rounding) * weight + (rounding + 4 * u) * out.abs()
    lse_bound = e + (keys * u + 8 * u) + 8 * u * lse.abs()
    return out_bound + 1e-30, lse_bound
