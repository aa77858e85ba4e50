"""The operators of the forward passes that the engine's sweeps go around, as
their users meet them, for timing and for comparing outputs.

Algorithm 1 evaluates the perturbed model twice a sample and keeps nothing but
two losses. Its forward passes need three operators, called through
``paper_2306_10015_amd.mezo``:

  attend  attention over a packed batch of documents (or over their key/value
          cache, for single tokens): grouped heads, causal with a visible
          prefix, scores capped by a tanh, a bias that grows with distance
  linear  a product in 8-bit floating point with a scale for each block of 128:
          activations quantized, weights in 8-bit storage or (``fresh``)
          quantized in the pass, as after every perturbation
  loss    the cross entropy of each token and the mean over the batch

A case's lengths of documents come from its own ``lens`` seed, so that its work
is known; the values come from the seed given to ``prepare``.
"""
from __future__ import annotations

import math
import random

import torch

#: False: the plain form, elementary torch operations. True: the framework's operators.
own = False

F8_BLOCK = 128
F8_MAX = 448.0


def listed():
    return [
        # the smallest set's model answers one token after a short prompt: all launch and latency
        {"name": "attend_token_opt125m_f32", "op": "attend", "dtype": "f32", "docs": 1, "lo": 37, "hi": 37, "new": 1,
         "capacity": 64, "heads": 12, "kv_heads": 12, "dim": 64, "prefix": False, "softcap": 0.0, "bias": False,
         "lens": 1},
        # a batch of answers in generation, an objective without a derivative: one token each over long caches
        {"name": "attend_tokens_cache_bf16", "op": "attend", "dtype": "bf16", "docs": 24, "lo": 500, "hi": 16384,
         "new": 1, "capacity": 16384, "heads": 32, "kv_heads": 8, "dim": 128, "prefix": False, "softcap": 0.0,
         "bias": False, "lens": 2},
        # a batch of classification prompts on the full-precision model, the prompt visible both ways
        {"name": "attend_prompts_opt125m_f32", "op": "attend", "dtype": "f32", "docs": 64, "lo": 11, "hi": 180,
         "new": 0, "capacity": 0, "heads": 12, "kv_heads": 12, "dim": 64, "prefix": True, "softcap": 0.0,
         "bias": False, "lens": 3},
        # a packed batch of ragged documents on the 1.3B shapes, a bias by distance
        {"name": "attend_packed_opt1.3b_bf16", "op": "attend", "dtype": "bf16", "docs": 16, "lo": 50, "hi": 2048,
         "new": 0, "capacity": 0, "heads": 32, "kv_heads": 32, "dim": 64, "prefix": True, "softcap": 0.0, "bias": True,
         "lens": 4},
        # one long document on the 6.7B shapes with capped scores: the largest attention
        {"name": "attend_long_opt6.7b_bf16", "op": "attend", "dtype": "bf16", "docs": 1, "lo": 8192, "hi": 8192,
         "new": 0, "capacity": 0, "heads": 32, "kv_heads": 32, "dim": 128, "prefix": False, "softcap": 30.0,
         "bias": False, "lens": 5},
        # one token through a projection of the smallest model
        {"name": "linear_token_opt125m", "op": "linear", "dtype": "f32", "out": "f32", "m": 1, "k": 768, "n": 768,
         "pad": 0, "fresh": False},
        # a batch of single tokens through the 6.7B model's wide layer: the weights' bytes
        {"name": "linear_tokens_opt6.7b", "op": "linear", "dtype": "bf16", "out": "bf16", "m": 24, "k": 4096,
         "n": 16384, "pad": 0, "fresh": False},
        # odd sizes, full precision in and out, activations that are a part of a wider array
        {"name": "linear_odd_f32", "op": "linear", "dtype": "f32", "out": "f32", "m": 1237, "k": 2050, "n": 8191,
         "pad": 14, "fresh": False},
        # a batch through weights that were perturbed just before and are quantized in the pass: the largest product
        {"name": "linear_perturbed_opt6.7b", "op": "linear", "dtype": "bf16", "out": "bf16", "m": 8192, "k": 16384,
         "n": 4096, "pad": 0, "fresh": True},
        # the verbalizer's token of one prompt over OPT's vocabulary
        {"name": "loss_token_f32", "op": "loss", "dtype": "f32", "t": 1, "v": 50272, "pad": 0, "skip": 0},
        # a batch of prompts of which a part counts, rows padded
        {"name": "loss_prompts_f32", "op": "loss", "dtype": "f32", "t": 1531, "v": 50272, "pad": 32, "skip": 410},
        # a batch of whole documents in bf16: the largest logits
        {"name": "loss_documents_bf16", "op": "loss", "dtype": "bf16", "t": 16384, "v": 50272, "pad": 0, "skip": 16},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every operator, type and option above, sizes over their
    logarithm, none costlier than the largest listed one of its operator."""
    op = rng.choice(["attend", "attend", "linear", "linear", "loss"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op == "loss":
        v = _log(rng, 100, 131072)
        t = _log(rng, 1, min(16384, 800_000_000 // v))
        return {"op": op, "dtype": dtype, "t": t, "v": v, "pad": rng.choice([0, 0, 3, 8, 32]),
                "skip": rng.choice([0, t // 3])}
    if op == "linear":
        m = rng.choice([_log(rng, 1, 64), _log(rng, 64, 8192)])
        k = _log(rng, 64, 16384)
        n = _log(rng, 64, min(50272, max(64, 8192 * 16384 * 4096 // (m * k))))
        if rng.random() < 0.5:
            k, n = (k + 63) // 64 * 64, (n + 63) // 64 * 64
        return {"op": op, "dtype": dtype, "out": rng.choice(["f32", "bf16", "bf16"]), "m": m, "k": k, "n": n,
                "pad": rng.choice([0, 0, 8, 24, 3]), "fresh": rng.random() < 0.3}
    dim = rng.choice([64, 64, 128, 128, 80, 40])
    kv_heads = rng.choice([1, 2, 4, 8, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    docs = _log(rng, 1, 64)
    new = rng.choice([0, 0, 1, rng.randint(2, 16)])
    # tokens of a document: at most 2^29 scores in a pass (the plain form holds them several times)
    top = math.sqrt(2.0 ** 29 / (docs * heads)) if not new else 2.0 ** 18 / docs
    hi = max(17, _log(rng, 17, max(18, min(16384, top))))
    return {"op": op, "dtype": dtype, "docs": docs, "lo": rng.choice([max(1, hi // 8), max(1, hi // 2), hi]), "hi": hi,
            "new": new, "capacity": hi + rng.choice([0, 1, 7]) if new else 0, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "prefix": rng.random() < 0.4, "softcap": rng.choice([0.0, 0.0, 30.0, 50.0]),
            "bias": rng.random() < 0.3, "lens": rng.randint(1, 1 << 30)}


_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- what the cases are made of ------------------------------------------------

def _documents(case):
    """[(q_first, q_len, k_first, k_len, prefix)] of a case, from its own seed. ``new``
    = 0: whole documents, packed one after another. Else the last ``new`` tokens of each
    (or all of a shorter one), over a cache of ``capacity`` rows a document."""
    r = random.Random(case["lens"])
    rows, at = [], 0
    for d in range(case["docs"]):
        n = r.randint(case["lo"], case["hi"])
        nq = min(n, case["new"]) if case["new"] else n
        prefix = r.randint(0, n) if case["prefix"] else 0
        rows.append((at, nq, d * case["capacity"] if case["new"] else at, n, prefix))
        at += nq
    return rows, at, case["docs"] * case["capacity"] if case["new"] else at


def _pairs(case):
    """Visible (query, key) pairs of a case, one head."""
    total = 0
    for _, nq, _, nk, prefix in _documents(case)[0]:
        first = nk - nq  # the first query's position
        # query i sees max(prefix, first + i + 1) keys
        flat = min(nq, max(0, prefix - first))
        total += flat * prefix + sum(range(first + flat + 1, nk + 1))
    return total


def _slopes(heads):
    """A geometric row of slopes, one for each head."""
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def _quantized(w):
    """Codes (bytes of e4m3) and scale exponents (bytes, biased by 127) of a
    matrix, in the layout of 8-bit storage: rows of codes padded with zeros to
    whole blocks, rows of scales padded with zeros to whole words."""
    codes, e = _to_f8(w.float())
    rows, blocks = e.shape
    scales = torch.zeros(rows, (blocks + 3) // 4 * 4, dtype=torch.uint8, device=w.device)
    scales[:, :blocks] = (e + 127).to(torch.uint8)
    return codes.view(torch.uint8).reshape(rows, -1), scales


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g)

    dt = _DTYPES[case["dtype"]]
    if case["op"] == "loss":
        logits = normal(case["t"], case["v"] + case["pad"], std=2.0).to(dt)[:, :case["v"]]
        targets = torch.randint(0, case["v"], (case["t"],), generator=g, device="cuda")
        skip = torch.randperm(case["t"], generator=g, device="cuda")[:case["skip"]]
        targets[skip] = -100
        return {"op": "loss", "logits": logits, "targets": targets}
    if case["op"] == "linear":
        x = normal(case["m"], case["k"] + case["pad"])
        # a few channels of a layer's input are much larger than the others
        loud = torch.randint(0, case["k"], (max(1, case["k"] // 256),), generator=g, device="cuda")
        x[:, loud] *= 20.0
        x = x.to(dt)[:, :case["k"]]
        w = normal(case["n"], case["k"], std=0.02)
        st = {"op": "linear", "x": x, "n": case["n"], "k": case["k"], "out": _DTYPES[case["out"]]}
        st["w"] = w.to(dt) if case["fresh"] else None
        # 8-bit weights: their buffers, filled where they are not quantized in the pass
        st["codes"], st["scales"] = _quantized(st["w"].new_zeros(w.shape) if case["fresh"] else w)
        return st
    rows, tq, tk = _documents(case)
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["new"]:
        q = normal(tq, h, d, std=1.5).to(dt)
        k, v = normal(tk, hk, d, std=1.5).to(dt), normal(tk, hk, d).to(dt)
    else:  # the three are parts of one projection's output
        qkv = normal(tq, h + 2 * hk, d, std=1.5).to(dt)
        q, k, v = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
    return {"op": "attend", "q": q, "k": k, "v": v, "table": torch.tensor(rows, dtype=torch.int64, device="cuda"),
            "max_q": max(r[1] for r in rows), "max_k": max(r[3] for r in rows), "softcap": case["softcap"],
            "slopes": torch.tensor(_slopes(h), dtype=torch.float32, device="cuda") if case["bias"] else None}


# ---- one pass --------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "loss":
        return _plain_loss(st["logits"], st["targets"])
    if st["op"] == "linear":
        if st["w"] is None:
            wv = st["codes"].view(torch.float8_e4m3fn).float().unflatten(1, (-1, F8_BLOCK))
            e = st["scales"][:, :wv.shape[1]].int() - 127
            wv = torch.ldexp(wv, e[:, :, None])
        else:
            wv = _f8_values(st["w"].float())
        xv = _f8_values(st["x"].float())
        return (xv.flatten(1) @ wv.flatten(1).t()).to(st["out"])
    return _plain_attend(st)


def _run_own(st):
    from paper_2306_10015_amd import mezo
    if st["op"] == "loss":
        return mezo.token_loss(st["logits"], st["targets"])
    if st["op"] == "linear":
        w = mezo.F8Matrix(st["codes"], st["scales"], st["n"], st["k"])
        if st["w"] is not None:
            mezo.f8_quantize(st["w"], out=w)
        return mezo.f8_linear(st["x"], w, st["out"])
    docs = mezo.Documents(st["table"], st["max_q"], st["max_k"])
    return mezo.attention(st["q"], st["k"], st["v"], docs, softcap=st["softcap"], slopes=st["slopes"], return_lse=True)


def _to_f8(w):
    """e4m3 codes [rows, blocks, 128] of float32 values, and their blocks'
    exponents: the least power of two that brings the block within 448."""
    w = torch.nn.functional.pad(w, (0, -w.shape[1] % F8_BLOCK)).unflatten(1, (-1, F8_BLOCK))
    m, x = torch.frexp(w.abs().amax(2))
    e = torch.where(m == 0, 0, x - 9 + (m > 0.875).int()).clamp(-127, 127)
    return torch.ldexp(w, -e[:, :, None]).to(torch.float8_e4m3fn), e


def _f8_values(w):
    codes, e = _to_f8(w)
    return torch.ldexp(codes.float(), e[:, :, None])


def _plain_loss(logits, targets):
    x = logits.float()
    top = x.amax(1, keepdim=True)
    lse = torch.log(torch.exp(x - top).sum(1)) + top[:, 0]
    counted = targets >= 0
    at = x.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    losses = torch.where(counted, lse - at, 0.0)
    return losses, losses.sum() / counted.sum().clamp(min=1)


def _plain_attend(st):
    """Every document padded to the longest one."""
    q, k, v, table = st["q"], st["k"], st["v"], st["table"]
    (tq, h, d), (tk, hk, _), b = q.shape, k.shape, table.shape[0]
    q0, nq, k0, nk, prefix = (c[:, None] for c in table.unbind(1))
    i = torch.arange(st["max_q"], device=q.device)
    j = torch.arange(st["max_k"], device=q.device)
    qi, kj = q0 + i, k0 + j
    qp = q.float()[qi.clamp(max=tq - 1)]  # [b, max_q, h, d]
    kp = k.float()[kj.clamp(max=tk - 1)].permute(0, 2, 3, 1).contiguous()  # [b, hk, d, max_k]
    vp = v.float()[kj.clamp(max=tk - 1)].permute(0, 2, 1, 3).contiguous()  # [b, hk, max_k, d]
    qp = qp.permute(0, 2, 1, 3).reshape(b, hk, -1, d)  # the heads of a group, one after another
    s = torch.matmul(qp, kp).mul_(1.0 / math.sqrt(d)).view(b, h, len(i), len(j))
    if st["softcap"]:
        s = torch.tanh_(s.div_(st["softcap"])).mul_(st["softcap"])
    pos = (nk - nq + i)[:, :, None]  # [b, max_q, 1]
    if st["slopes"] is not None:
        s -= st["slopes"][:, None, None] * (pos - j).abs()[:, None]
    seen = ((j <= pos) | (j < prefix[:, :, None])) & (j < nk[:, :, None])
    s.masked_fill_(~seen[:, None], -math.inf)
    top = s.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(3)
    o = torch.matmul(p.view(b, hk, -1, len(j)), vp).view(b, h, len(i), d)
    o = torch.where(total[..., None] > 0, o / total[..., None], 0.0)
    lse = top[..., 0] + torch.log(total)
    # padded queries go to a row past the end
    to = torch.where(i < nq, qi, tq).flatten()
    out = torch.zeros(tq + 1, h, d, dtype=torch.float32, device=q.device)
    out[to] = o.permute(0, 2, 1, 3).reshape(-1, h, d)
    out_lse = torch.zeros(tq + 1, h, dtype=torch.float32, device=q.device)
    out_lse[to] = lse.permute(0, 2, 1).reshape(-1, h)
    return out[:tq].to(q.dtype), out_lse[:tq]


# ---- cost and definition -----------------------------------------------------------

def work(case):
    size = _DTYPES[case["dtype"]].itemsize
    if case["op"] == "loss":
        rows = case["t"] - case["skip"]
        return {"bytes": rows * case["v"] * size + case["t"] * 12 + 4, "flops": 4 * rows * case["v"]}
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        weights = n * k * size if case["fresh"] else n * (k + (k + F8_BLOCK - 1) // F8_BLOCK)
        return {"bytes": m * k * size + weights + m * n * _DTYPES[case["out"]].itemsize, "flops": 2 * m * k * n}
    rows, tq, _ = _documents(case)
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    keys = sum(r[3] for r in rows)
    return {"bytes": (2 * tq * h + 2 * keys * hk) * d * size + tq * h * 4, "flops": 4 * d * h * _pairs(case)}


def _exact_f8(w):
    """The values that 8-bit storage holds for w, in 64 bits."""
    w = w.double()
    out = torch.zeros_like(w)
    for at in range(0, w.shape[1], F8_BLOCK):
        part = w[:, at:at + F8_BLOCK]
        top = part.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, F8_MAX) / F8_MAX))
        # (log2 rounds: the least exponent that holds the block, by comparison)
        e = torch.where(top > F8_MAX * torch.exp2(e), e + 1, e)
        e = torch.where(top <= F8_MAX * torch.exp2(e - 1), e - 1, e)
        e = torch.where(top > 0, e, 0.0).clamp(-127, 127)
        x = part / torch.exp2(e)
        # four significant bits, the grid of 2^-9 below 2^-6
        step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, at:at + F8_BLOCK] = torch.round(x / step) * step * torch.exp2(e)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "loss":
        losses = torch.zeros(case["t"], dtype=torch.float64, device="cuda")
        for a in range(0, case["t"], 1024):
            x, t = st["logits"][a:a + 1024].double(), st["targets"][a:a + 1024]
            own_logit = x[torch.arange(len(t), device="cuda"), t.clamp(min=0)]
            losses[a:a + 1024] = torch.where(t >= 0, torch.logsumexp(x, 1) - own_logit, 0.0)
        return losses, losses.sum() / max(1, case["t"] - case["skip"])
    if case["op"] == "linear":
        if case["fresh"]:
            w = _exact_f8(st["w"])
        else:
            byte = st["codes"][:, :case["k"]].int()
            mant, ex = (byte & 7).double(), (byte >> 3) & 15
            w = torch.where(ex > 0, (8 + mant) * torch.exp2(ex.double() - 10), mant * 2.0 ** -9)
            w = torch.where(byte > 127, -w, w)
            w *= torch.exp2(st["scales"].double() - 127).repeat_interleave(F8_BLOCK, 1)[:, :case["k"]]
        return _exact_f8(st["x"]) @ w.t().contiguous()
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    (tq, h, d), group = q.shape, q.shape[1] // k.shape[1]
    out = torch.zeros(tq, h, d, dtype=torch.float64, device="cuda")
    out_lse = torch.zeros(tq, h, dtype=torch.float64, device="cuda")
    for q0, nq, k0, nk, prefix in _documents(case)[0]:
        at = torch.arange(nk - nq, nk, device="cuda")[:, None]
        key = torch.arange(nk, device="cuda")[None, :]
        hidden = (key > at) & (key >= prefix)
        for head in range(h):
            s = q[q0:q0 + nq, head] @ k[k0:k0 + nk, head // group].t().contiguous() / math.sqrt(d)
            if case["softcap"]:
                s = case["softcap"] * torch.tanh(s / case["softcap"])
            if case["bias"]:
                s = s - st["slopes"][head].double() * (at - key).abs()
            s = s.masked_fill(hidden, -math.inf)
            out_lse[q0:q0 + nq, head] = torch.logsumexp(s, 1)
            out[q0:q0 + nq, head] = torch.softmax(s, 1) @ v[k0:k0 + nk, head // group]
    return out, out_lse
