"""Generation over a paged cache on 4-bit weights, for timing and for comparing
outputs.

An objective without a derivative is scored on answers that the perturbed model
generates. A step of generation needs three operators beside those of a whole
document's pass, called through ``paper_2306_10015_amd.mezo``:

  append   new keys and values into a paged cache, turned by their positions on
           the way, the queries turned by the same call
  attend   attention of a document's last tokens over its pages: a single token,
           a chunk of a prompt, or a tree of drafted tokens
  product  activations times weights in 4-bit storage, which are never written out

A case's lengths and trees come from its own ``lens`` seed, so that its work is
known; values and the order of the pages come from the seed given to ``prepare``.
"""
from __future__ import annotations

import math
import random

import torch

#: False: the plain form, elementary torch operations. True: the framework's operators.
own = False

#: NF4's values, and the elements that share a scale.
NF4 = [-1.0, -0.6961928009986877, -0.5250730514526367, -0.39491748809814453, -0.28444138169288635, -0.18477343022823334,
       -0.09105003625154495, 0.0, 0.07958029955625534, 0.16093020141124725, 0.24611230194568634, 0.33791524171829224,
       0.44070982933044434, 0.5626170039176941, 0.7229568362236023, 1.0]
BLOCK = 64


def listed():
    return [
        # one token of the smallest set's model into the cache: all launch and latency
        {"name": "append_token_opt125m_f32", "op": "append", "dtype": "f32", "docs": 1, "lo": 38, "hi": 38, "new": 1,
         "tree": False, "page": 16, "heads": 12, "kv_heads": 12, "dim": 64, "rot": 64, "interleaved": False, "lens": 1},
        # a batch of answers in generation: one token each, half of a head's columns turned
        {"name": "append_tokens_bf16", "op": "append", "dtype": "bf16", "docs": 24, "lo": 500, "hi": 2048, "new": 1,
         "tree": False, "page": 16, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 64, "interleaved": True, "lens": 2},
        # a batch of whole prompts on the 6.7B shapes: the largest append
        {"name": "append_prompts_opt6.7b_bf16", "op": "append", "dtype": "bf16", "docs": 16, "lo": 50, "hi": 2048,
         "new": 0, "tree": False, "page": 32, "heads": 32, "kv_heads": 32, "dim": 128, "rot": 128,
         "interleaved": False, "lens": 3},
        # the smallest set's model answers one token after a short prompt
        {"name": "attend_token_opt125m_f32", "op": "attend", "dtype": "f32", "docs": 1, "lo": 37, "hi": 37, "new": 1,
         "tree": False, "page": 16, "heads": 12, "kv_heads": 12, "dim": 64, "prefix": False, "softcap": 0.0,
         "bias": False, "lens": 4},
        # a batch of answers in generation: one token each over long caches of small pages
        {"name": "attend_tokens_bf16", "op": "attend", "dtype": "bf16", "docs": 24, "lo": 500, "hi": 16384, "new": 1,
         "tree": False, "page": 16, "heads": 32, "kv_heads": 8, "dim": 128, "prefix": False, "softcap": 0.0,
         "bias": False, "lens": 2},
        # eight answers, each with a tree of drafted tokens that is checked in one pass
        {"name": "attend_trees_bf16", "op": "attend", "dtype": "bf16", "docs": 8, "lo": 500, "hi": 8192, "new": 61,
         "tree": True, "page": 64, "heads": 32, "kv_heads": 8, "dim": 128, "prefix": False, "softcap": 0.0,
         "bias": False, "lens": 5},
        # chunks of long prompts on the 6.7B shapes, over what is in the cache already: the largest attention
        {"name": "attend_chunks_opt6.7b_bf16", "op": "attend", "dtype": "bf16", "docs": 4, "lo": 600, "hi": 8192,
         "new": 1000, "tree": False, "page": 32, "heads": 32, "kv_heads": 32, "dim": 128, "prefix": False,
         "softcap": 0.0, "bias": False, "lens": 6},
        # one token through a projection of the smallest model
        {"name": "product_token_opt125m_f32", "op": "product", "dtype": "f32", "out": "f32", "m": 1, "k": 768,
         "n": 768, "pad": 0},
        # one token through the 6.7B model's wide layer: the weights' bytes
        {"name": "product_token_opt6.7b", "op": "product", "dtype": "bf16", "out": "bf16", "m": 1, "k": 4096,
         "n": 16384, "pad": 0},
        # a batch of single tokens through the way back
        {"name": "product_tokens_opt6.7b", "op": "product", "dtype": "bf16", "out": "bf16", "m": 24, "k": 16384,
         "n": 4096, "pad": 0},
        # full precision, odd sizes (blocks run over the ends of rows), activations that are a part of a wider array
        {"name": "product_odd_f32", "op": "product", "dtype": "f32", "out": "f32", "m": 1237, "k": 2050, "n": 8191,
         "pad": 14},
        # a batch of whole documents: the largest product
        {"name": "product_documents_opt6.7b", "op": "product", "dtype": "bf16", "out": "bf16", "m": 8192, "k": 16384,
         "n": 4096, "pad": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every operator, type and option above, sizes over their
    logarithm, none costlier than the largest listed one of its operator."""
    op = rng.choice(["append", "attend", "attend", "product", "product"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op == "product":
        m = rng.choice([1, _log(rng, 2, 64), _log(rng, 64, 8192)])
        k = _log(rng, 64, 16384)
        n = _log(rng, 64, min(50272, max(64, 8192 * 16384 * 4096 // (m * k))))
        if rng.random() < 0.6:
            k = (k + 63) // 64 * 64
        return {"op": op, "dtype": dtype, "out": rng.choice([dtype, dtype, "f32", "bf16"]), "m": m, "k": k, "n": n,
                "pad": rng.choice([0, 0, 8, 24, 3])}
    dim = rng.choice([64, 64, 128, 128, 80, 40])
    kv_heads = rng.choice([1, 2, 4, 8, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    docs = _log(rng, 1, 64)
    page = rng.choice([8, 16, 16, 32, 64, 256])
    if op == "append":
        new = rng.choice([0, 1, 1, rng.randint(2, 64)])
        top = 6 * 2.0 ** 17 / docs / (heads + 2 * kv_heads)
        hi = max(17, _log(rng, 17, max(18, min(8192, top))))
        return {"op": op, "dtype": dtype, "docs": docs, "lo": rng.choice([max(1, hi // 8), hi]), "hi": hi, "new": new,
                "tree": new > 1 and rng.random() < 0.4, "page": page, "heads": heads, "kv_heads": kv_heads,
                "dim": dim, "rot": rng.choice([dim, dim, dim // 2, 0]), "interleaved": rng.random() < 0.5,
                "lens": rng.randint(1, 1 << 30)}
    new = rng.choice([1, 1, rng.randint(2, 16), _log(rng, 16, 512), 0])
    # keys of a document: at most 2^28 scores in a pass (the plain form holds them several times)
    top = math.sqrt(2.0 ** 28 / (docs * heads)) if not new else min(2.0 ** 28 / (docs * heads * new), 2.0 ** 18 / docs)
    hi = max(17, _log(rng, 17, max(18, min(16384, top))))
    tree = new > 1 and rng.random() < 0.6
    return {"op": op, "dtype": dtype, "docs": docs, "lo": rng.choice([max(1, hi // 8), max(1, hi // 2), hi]), "hi": hi,
            "new": new, "tree": tree, "page": page, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "prefix": not tree and rng.random() < 0.3, "softcap": rng.choice([0.0, 0.0, 30.0, 50.0]),
            "bias": not tree and rng.random() < 0.3, "lens": rng.randint(1, 1 << 30)}


_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- what the cases are made of ------------------------------------------------

def _documents(case):
    """([(q_first, q_len, first entry, k_len, prefix)], tokens, entries, parents) of
    a case, from its own seed: the last ``new`` tokens of each document (0: all), and
    for trees each token's parent among its document's new ones (-1: the last token
    before them)."""
    r = random.Random(case["lens"])
    rows, at, entry, parents = [], 0, 0, []
    for _ in range(case["docs"]):
        n = r.randint(case["lo"], case["hi"])
        nq = min(n, case["new"]) if case["new"] else n
        prefix = r.randint(0, n) if case.get("prefix") else 0
        rows.append((at, nq, entry, n, prefix))
        at += nq
        entry += (n + case["page"] - 1) // case["page"]
        if case["tree"]:
            parents.append([-1 if t == 0 else r.randint(max(-1, t - 9), t - 1) for t in range(nq)])
    return rows, at, entry, parents


def _tree(parents):
    """([64-bit words] of each token: which of its document's new tokens it follows,
    itself too; depths), as host lists."""
    words = (max(map(len, parents)) + 63) // 64
    masks, depths = [], []
    for tree in parents:
        first = len(masks)
        for t, p in enumerate(tree):
            masks.append((masks[first + p] if p >= 0 else 0) | 1 << t)
            depths.append(depths[first + p] + 1 if p >= 0 else 0)
    low = (1 << 64) - 1
    split = [[m >> 64 * w & low for w in range(words)] for m in masks]
    return [[w - (1 << 64) if w >> 63 else w for w in row] for row in split], depths


def _pairs(case):
    """Visible (query, key) pairs of a case, one head."""
    rows, _, _, parents = _documents(case)
    if case["tree"]:
        depths, total, at = _tree(parents)[1], 0, 0
        for _, nq, _, nk, _ in rows:
            total += nq * (nk - nq) + sum(d + 1 for d in depths[at:at + nq])
            at += nq
        return total
    total = 0
    for _, nq, _, nk, prefix in rows:
        first = nk - nq  # the first query's position
        # query i sees max(prefix, first + i + 1) keys
        flat = min(nq, max(0, prefix - first))
        total += flat * prefix + sum(range(first + flat + 1, nk + 1))
    return total


def _slopes(heads):
    """A geometric row of slopes, one for each head."""
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g)

    dt = _DTYPES[case["dtype"]]
    if case["op"] == "product":
        m, k, n = case["m"], case["k"], case["n"]
        x = normal(m, k + case["pad"])
        # a few channels of a layer's input are much larger than the others
        loud = torch.randint(0, k, (max(1, k // 256),), generator=g, device="cuda")
        x[:, loud] *= 20.0
        values = torch.tensor(NF4, device="cuda")
        w = normal((n * k + BLOCK - 1) // BLOCK, BLOCK, std=0.02)
        absmax = w.abs().amax(1)
        codes = torch.bucketize(w / absmax[:, None], (values[1:] + values[:-1]) / 2).to(torch.uint8).flatten()
        codes = codes[:n * k + n * k % 2]
        return {"op": "product", "x": x.to(dt)[:, :k], "codes": codes[::2] | codes[1::2] << 4, "absmax": absmax,
                "n": n, "k": k, "out": _DTYPES[case["out"]]}
    rows, tokens, entries, parents = _documents(case)
    h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    n_pages = entries + entries // 8 + 1  # of some the documents have no use
    st = {"op": case["op"], "table": torch.tensor(rows, dtype=torch.int64, device="cuda"),
          "pages": torch.randperm(n_pages, generator=g, device="cuda")[:entries].int(),
          "max_q": max(r[1] for r in rows), "max_k": max(r[3] for r in rows), "mask": None, "positions": None,
          "k_pages": normal(n_pages, page, hk, d, std=1.5).to(dt), "v_pages": normal(n_pages, page, hk, d).to(dt)}
    if case["tree"]:
        mask, depths = _tree(parents)
        st["mask"] = torch.tensor(mask, dtype=torch.int64, device="cuda")
        first = [nk - nq for _, nq, _, nk, _ in rows for _ in range(nq)]
        st["positions"] = torch.tensor([a + b for a, b in zip(first, depths)], dtype=torch.int64, device="cuda")
    if case["op"] == "append":  # the three are parts of one projection's output
        qkv = normal(tokens, h + 2 * hk, d).to(dt)
        st.update(q=qkv[:, :h], k=qkv[:, h:h + hk], v=qkv[:, h + hk:], interleaved=case["interleaved"], freqs=None)
        if case["rot"]:
            exponent = torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"]
            st["freqs"] = (10000.0 ** -exponent).float()
        return st
    st.update(q=normal(tokens, h, d, std=1.5).to(dt), softcap=case["softcap"],
              slopes=torch.tensor(_slopes(h), dtype=torch.float32, device="cuda") if case["bias"] else None)
    return st


# ---- one pass --------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"append": _plain_append, "attend": _plain_attend, "product": _plain_product}[st["op"]](st)


def _run_own(st):
    from paper_2306_10015_amd import mezo
    if st["op"] == "product":
        return mezo.nf4_linear(st["x"], mezo.NF4Tensor(st["codes"], st["absmax"], st["n"] * st["k"]), st["out"])
    cache = mezo.PagedCache(st["k_pages"], st["v_pages"], st["pages"])
    docs = mezo.Documents(st["table"], st["max_q"], st["max_k"])
    if st["op"] == "append":
        q = mezo.cache_append(st["k"], st["v"], cache, docs, q=st["q"], freqs=st["freqs"], positions=st["positions"],
                              interleaved=st["interleaved"])
        return q, st["k_pages"], st["v_pages"]
    return mezo.paged_attention(st["q"], cache, docs, tree=st["mask"], softcap=st["softcap"], slopes=st["slopes"],
                                return_lse=True)


def _plain_product(st):
    n, k = st["n"], st["k"]
    values = torch.tensor(NF4, device="cuda")
    codes = torch.stack((st["codes"] & 15, st["codes"] >> 4), 1).flatten()[:n * k]
    w = values[codes.int()]
    w = torch.nn.functional.pad(w, (0, -len(w) % BLOCK)).view(-1, BLOCK) * st["absmax"][:, None]
    w = w.flatten()[:n * k].view(n, k).to(st["x"].dtype)
    return (st["x"].float() @ w.float().t()).to(st["out"])


def _places(st):
    """Of every new token: its place in its document, and that place's row of the cache."""
    q0, nq, first, nk, _ = st["table"].unbind(1)
    tokens, page = st["q"].shape[0], st["k_pages"].shape[1]
    doc = torch.repeat_interleave(torch.arange(len(nq), device=nq.device), nq, output_size=tokens)
    place = torch.arange(tokens, device=nq.device) - q0[doc] + (nk - nq)[doc]
    return place, st["pages"][first[doc] + place // page].long() * page + place % page


def _turned(x, cos, sin, interleaved):
    """x [tokens, heads, dim] with its first columns turned, pair by pair."""
    half = cos.shape[1]
    x = x.float()
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    c, s = cos[:, None], sin[:, None]
    pair = (a * c - b * s, a * s + b * c)
    out = x.clone()
    out[..., :2 * half] = torch.stack(pair, 3).flatten(2) if interleaved else torch.cat(pair, 2)
    return out


def _plain_append(st):
    place, row = _places(st)
    q, k, dt = st["q"], st["k"], st["q"].dtype
    if st["freqs"] is not None:
        pos = place if st["positions"] is None else st["positions"]
        angle = pos.double()[:, None] * st["freqs"].double()
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        q, k = _turned(q, cos, sin, st["interleaved"]), _turned(k, cos, sin, st["interleaved"])
    st["k_pages"].flatten(0, 1)[row] = k.to(dt)
    st["v_pages"].flatten(0, 1)[row] = st["v"]
    return q.to(dt).contiguous(), st["k_pages"], st["v_pages"]


def _plain_attend(st):
    """Every document's pages gathered, padded to the longest one."""
    q, table = st["q"], st["table"]
    page, hk = st["k_pages"].shape[1:3]
    (tq, h, d), b = q.shape, table.shape[0]
    q0, nq, first, nk, prefix = (c[:, None] for c in table.unbind(1))
    i = torch.arange(st["max_q"], device=q.device)
    j = torch.arange(st["max_k"], device=q.device)
    at = torch.where(j < nk, first + j // page, 0)
    kj = st["pages"][at].long() * page + j % page
    qi = q0 + i
    qp = q.float()[qi.clamp(max=tq - 1)]  # [b, max_q, h, d]
    kp = st["k_pages"].flatten(0, 1)[kj].float().permute(0, 2, 3, 1).contiguous()  # [b, hk, d, max_k]
    vp = st["v_pages"].flatten(0, 1)[kj].float().permute(0, 2, 1, 3).contiguous()  # [b, hk, max_k, d]
    qp = qp.permute(0, 2, 1, 3).reshape(b, hk, -1, d)  # the heads of a group, one after another
    s = torch.matmul(qp, kp).mul_(1.0 / math.sqrt(d)).view(b, h, len(i), len(j))
    if st["softcap"]:
        s = torch.tanh_(s.div_(st["softcap"])).mul_(st["softcap"])
    pos = (nk - nq + i)[:, :, None]  # [b, max_q, 1]
    if st["slopes"] is not None:
        s -= st["slopes"][:, None, None] * (pos - j).abs()[:, None]
    seen = (j <= pos) | (j < prefix[:, :, None])
    if st["mask"] is not None:
        t = (j - (nk - nq))[:, None, :]  # which of the new tokens a key is
        word = st["mask"][qi.clamp(max=tq - 1)]  # [b, max_q, words]
        word = word.gather(2, (t >> 6).clamp(0, word.shape[2] - 1).expand(-1, len(i), -1))
        seen = (t < 0) | (word >> (t & 63) & 1).bool()
    seen &= (j < nk)[:, None]
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
    if case["op"] == "product":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": m * k * size + (n * k + 1) // 2 + (n * k + BLOCK - 1) // BLOCK * 4 +
                m * n * _DTYPES[case["out"]].itemsize, "flops": 2 * m * k * n}
    rows, tokens, entries, _ = _documents(case)
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "append":
        return {"bytes": 2 * tokens * (h + 2 * hk) * d * size, "flops": 3 * tokens * (h + hk) * case["rot"]}
    keys = sum(r[3] for r in rows)
    return {"bytes": (2 * tokens * h + 2 * keys * hk) * d * size + entries * 4 + tokens * h * 4,
            "flops": 4 * d * h * _pairs(case)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "product":
        n, k = case["n"], case["k"]
        nibbles = torch.empty(2 * len(st["codes"]), dtype=torch.long, device="cuda")
        nibbles[0::2], nibbles[1::2] = st["codes"] % 16, st["codes"] // 16
        w = torch.tensor(NF4, dtype=torch.float64, device="cuda").float().double()[nibbles[:n * k]]
        # (the product of two floats is exact in 64 bits)
        w *= st["absmax"].double().repeat_interleave(BLOCK)[:n * k]
        w = w.float().to(st["x"].dtype).double().view(n, k)
        return st["x"].double() @ w.t().contiguous()
    rows, tokens, _, parents = _documents(case)
    h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    kc, vc = st["k_pages"].double().flatten(0, 1), st["v_pages"].double().flatten(0, 1)
    pages = st["pages"].tolist()

    def cache_rows(first, lo, hi):
        return torch.tensor([pages[first + j // page] * page + j % page for j in range(lo, hi)], dtype=torch.long,
                            device="cuda")

    if case["op"] == "append":
        qo = st["q"].double().contiguous()
        for q0, nq, first, nk, _ in rows:
            part, to = slice(q0, q0 + nq), cache_rows(first, nk - nq, nk)
            pos = torch.arange(nk - nq, nk, device="cuda") if st["positions"] is None else st["positions"][part]
            kr = st["k"][part].double()
            if case["rot"]:
                # a pair as a complex number, turned by the unit one of its angle
                unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(nq, case["rot"] // 2),
                                   torch.outer(pos.double(), st["freqs"].double()))[:, None]
                for x in (qo[part], kr):
                    y = x[..., :case["rot"]]
                    if case["interleaved"]:
                        y.copy_(torch.view_as_real(torch.view_as_complex(y.unflatten(2, (-1, 2)).contiguous()) * unit)
                                .flatten(2))
                    else:
                        z = torch.complex(*(p.contiguous() for p in y.chunk(2, 2))) * unit
                        y.copy_(torch.cat((z.real, z.imag), 2))
            kc[to], vc[to] = kr, st["v"][part].double()
        return qo, kc.view(st["k_pages"].shape), vc.view(st["v_pages"].shape)
    q = st["q"].double()
    out = torch.zeros(tokens, h, d, dtype=torch.float64, device="cuda")
    out_lse = torch.zeros(tokens, h, dtype=torch.float64, device="cuda")
    for doc, (q0, nq, first, nk, prefix) in enumerate(rows):
        at = torch.arange(nk - nq, nk, device="cuda")[:, None]
        key = torch.arange(nk, device="cuda")[None, :]
        hidden = (key > at) & (key >= prefix)
        if case["tree"]:
            follows = torch.zeros(nq, nq, dtype=torch.bool)
            for t, p in enumerate(parents[doc]):
                if p >= 0:
                    follows[t] = follows[p]
                follows[t, t] = True
            hidden = torch.cat((torch.zeros(nq, nk - nq, dtype=torch.bool), ~follows), 1).cuda()
        row = cache_rows(first, 0, nk)
        for head in range(h):
            k, v = kc[row, head // (h // hk)], vc[row, head // (h // hk)]
            s = q[q0:q0 + nq, head] @ k.t().contiguous() / math.sqrt(d)
            if case["softcap"]:
                s = case["softcap"] * torch.tanh(s / case["softcap"])
            if case["bias"]:
                s = s - st["slopes"][head].double() * (at - key).abs()
            s = s.masked_fill(hidden, -math.inf)
            out_lse[q0:q0 + nq, head] = torch.logsumexp(s, 1)
            out[q0:q0 + nq, head] = torch.softmax(s, 1) @ v
    return out, out_lse
