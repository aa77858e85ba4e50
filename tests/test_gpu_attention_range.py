"""Attention on the GPU at the ends of its range: caps of any size, scores and
values near the ends of their types, split documents with every score function,
and what tokens that are not finite cost. Against the plain reference in 64 bits
(attention_ref.py); the bars come from the arithmetic (bounds)."""
import math

import pytest

import attention_ref
from test_gpu_attention import DTYPES, table, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def bounds(out, lse, weight, q, k, dtype, keys, scale, softcap, slopes):
    """How far out and lse may be off. With u = 2^-24: a product of dim terms is off by
    u (dim + 8) of the sum of their sizes; a cap is applied to 16 u of the score itself
    and, up to 66 and for bf16, to 8 u of the cap; a bias by distance to 4 u of itself;
    the difference from the reference and exp2 to 8 u of the score. No term grows with
    a larger cap."""
    u = 2.0 ** -24
    heads, dim, group = q.shape[1], q.shape[2], q.shape[1] // k.shape[1]
    scale = 1.0 / math.sqrt(dim) if scale is None else abs(scale)
    qa, ka = q.cpu().double().abs(), k.cpu().double().abs()
    raw = max(float((qa[:, h] @ ka[:, h // group].t()).max()) for h in range(heads)) * scale
    top = min(raw, softcap) if softcap else raw
    e = u * (dim + 8) * (raw if math.isfinite(raw) else 0.0)
    if softcap:
        e += 16 * u * top + 8 * u * min(softcap, 66.6)
    if slopes is not None:
        far = float(slopes.abs().max()) * keys
        e += 4 * u * far
        top += far
    e += 8 * u * top + 4 * u
    rounding = 2.0 ** -8 if str(dtype) == "torch.bfloat16" else 0.0
    return ((2 * e + 2 * keys * u + rounding) * weight + (rounding + 4 * u) * out.abs(),
            e + (keys * u + 8 * u) + 8 * u * lse.abs())


def check(mz, q, k, v, rows, causal=True, scale=None, softcap=0.0, slopes=None, max_k=None, floor=2.0 ** -126):
    import torch
    docs = mz.Documents(torch.tensor(rows, dtype=torch.int64, device="cuda"), max(r[1] for r in rows),
                        max(r[3] for r in rows) if max_k is None else max_k)
    out, lse = mz.attention(q, k, v, docs, causal=causal, scale=scale, softcap=softcap, slopes=slopes, return_lse=True)
    want, want_lse, weight = attention_ref.attention(q, k, v, rows, causal, scale, softcap, slopes)
    ob, lb = bounds(want, want_lse, weight, q, k, q.dtype, max(r[3] for r in rows), scale, softcap, slopes)
    off = (out.cpu().double() - want).abs()
    ob += floor
    assert bool((off <= ob).all()), float((off / ob).max())
    off = (lse.cpu().double() - want_lse).abs()
    off[lse.cpu().double() == want_lse] = 0.0  # (infinities)
    assert bool((off <= lb).all()), float((off / lb).max())
    return out, lse


# ---- caps of any size ----------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cap", [1e-40, 1e-12, 0.5, 66.0, 67.0, 100.0, 1e4, 1e6, 1e8, 1e30, 3.4e38])
@pytest.mark.parametrize("bias", [False, True])
def test_caps_of_any_size(mz, cap, bias, dtype):
    """A cap far above the scores leaves them as they are, one far below takes them to 0."""
    import torch
    slopes = torch.tensor([0.5, 0.03, 0.0, -0.01], device="cuda") if bias else None
    q, k, v = tensors(150, 150, 4, 2, 64, dtype)
    q = q * 3
    k[3] = 0  # a score of 0
    check(mz, q, k, v, table([150], prefix=[10]), softcap=cap, slopes=slopes)
    check(mz, q[:2], k, v, table([2], [150]), softcap=cap, slopes=slopes)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cap", [100.0, 1e4, 1e8])
def test_large_caps_and_large_scores(mz, cap, dtype):
    """Scores of the size of the cap, where neither end of the tanh holds."""
    q, k, v = tensors(130, 130, 2, 1, 64, dtype)
    check(mz, q, k, v, table([130]), softcap=cap, scale=cap / 30)
    check(mz, q[:1], k, v, table([1], [130]), softcap=cap, scale=cap / 30)


# ---- values near the ends of their types ------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cap", [30.0, 50.0, 66.0])
@pytest.mark.parametrize("size", [1e-30, 1.0, 1e30])
@pytest.mark.parametrize("sign", [-1, 1])
def test_saturated_caps_keep_the_values_digits(mz, sign, size, cap, dtype):
    """All scores at one end of the cap: as good a softmax as any other, for values of
    any size."""
    q, k, v = tensors(150, 150, 2, 2, 64, dtype)
    q, k = q * 0.01 + 4.0, k * 0.01 + sign * 4.0
    check(mz, q, k, v * size, table([150]), softcap=cap)
    check(mz, q[:40], k, v[:150] * size, table([40], [150]), softcap=cap)
    check(mz, q[:1], k, v[:150] * size, table([1], [150]), softcap=cap)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cap", [20.0, 50.0, 66.0])
@pytest.mark.parametrize("size", [1e-30, 1.0, 1e12])
@pytest.mark.parametrize("at", [1, 63, 64, 100, 149])
def test_caps_from_one_end_to_the_other(mz, at, size, cap, dtype):
    """Keys of score -cap, then one of +cap, then -cap again: the rows before it are
    theirs, the rows after it its."""
    q, k, v = tensors(150, 150, 2, 2, 64, dtype)
    q, k = q * 0.01 + 4.0, k * 0.01 - 4.0
    k[at] += 8.0
    check(mz, q, k, v * size, table([150]), softcap=cap)
    check(mz, q, k, v * size, table([150]), softcap=cap, causal=False)


# ---- tokens that are not finite: what they cost -----------------------------------

def seconds(call, passes=5):
    import torch
    call()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(passes):
        call()
    end.record()
    end.synchronize()
    return start.elapsed_time(end) / 1000 / passes


@pytest.mark.parametrize("which,most", [("q", 40), ("k", 40), ("v", 400)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_tokens_that_are_not_finite_do_not_stall_a_pass(mz, bad, which, most):
    """A token that every row sees (or every query) is not finite, as when a model
    diverges, and every row is computed a second time. Queries and keys: a row ends at
    its first 64 keys, a few us of latency for each of a wave's 32 rows, where the pass
    takes 30 us or so. Values: about 15 instructions of a wave a row and key, where the
    pass has one for 7 rows and keys, and little to hide their latency behind."""
    import torch
    q, k, v = tensors(2048, 2048, 8, 8, 64, "bf16")
    docs = mz.Documents.of([2048])
    clean = seconds(lambda: mz.attention(q, k, v, docs))
    if which == "q":
        q[:, :, 5] = bad
    else:
        (k if which == "k" else v)[0, :, 5] = bad
    spent = seconds(lambda: mz.attention(q, k, v, docs))
    print(f"clean {clean * 1e6:.0f} us, {which} {bad}: {spent * 1e6:.0f} us")
    out = mz.attention(q, k, v, docs).float()
    if which != "v" and bad > 0:  # (a score of -inf takes no part)
        out = out[~torch.isfinite(out).all(2)]
        assert len(out) > 0
    assert not bool(torch.isfinite(out[..., 5]).any())
    if which == "v":
        assert bool(torch.isfinite(out[..., :5]).all())
    assert spent <= most * clean


# ---- scores and values near the largest float --------------------------------------

SHAPES = [(70, 70), (1, 300), (5, 300), (1, 3000), (129, 2600)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,nk", SHAPES)
@pytest.mark.parametrize("size", [-3e38, -2.5e38, 2.5e38, 3e38])
def test_scores_near_the_largest_float(mz, size, nq, nk, dtype):
    """Scores that are finite, but not in units of log 2: a row of equal ones is the mean
    of its values, and one that is larger takes it all."""
    import torch
    q, k, v = tensors(nq, nk, 2, 2, 64, dtype)
    q.zero_()
    k.zero_()
    q[..., 0] = 1
    rows = table([nq], [nk])
    docs = mz.Documents.of([nq], [nk])
    # a mean of up to 2600 terms rounded to bf16 each, then itself
    bar = 2.0 ** -6 if dtype == "bf16" else 2e-4
    for one in (False, True):
        k[..., 0] = size
        if one:
            k[nk // 2, :, 0] = size * (0.9 if size < 0 else 1.1)
        out, lse = mz.attention(q, k, v, docs, scale=1.0, return_lse=True)
        want, want_lse, _ = attention_ref.attention(q, k, v, rows, scale=1.0)
        assert float((out.cpu().double() - want).abs().max()) <= bar
        assert float(((lse.cpu().double() - want_lse) / size).abs().max()) <= 1e-6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,nk", SHAPES)
@pytest.mark.parametrize("softcap", [0.0, 30.0])
def test_values_near_the_largest_float(mz, softcap, nq, nk, dtype):
    """A mean of values is no larger than they are."""
    q, k, v = tensors(nq, nk, 2, 2, 64, dtype)
    v = (v.sign() * (1 - v.abs().clamp(max=0.9)) * 3.3e38).to(v.dtype)
    v[:, :, :8] = 3.3e38
    check(mz, q, k, v, table([nq], [nk]), softcap=softcap)


# ---- split documents -----------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq", [1, 40, 129])
@pytest.mark.parametrize("softcap,bias,prefix", [(30.0, False, 0), (0.0, True, 0), (5.0, True, 0), (100.0, False, 0),
                                                 (0.0, False, 2590), (30.0, False, 2590)])
def test_split_documents_with_every_score_function(mz, softcap, bias, prefix, nq, dtype):
    import torch
    n = 2600
    slopes = torch.tensor([0.1, 0.003, 0.0, -0.002], device="cuda") if bias else None
    q, k, v = tensors(2 * nq, n + 700, 4, 2, 64, dtype)
    check(mz, q, k, v, table([nq] * 2, [n, 700], [prefix, 0]), softcap=softcap, slopes=slopes)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq", [1, 40, 129])
@pytest.mark.parametrize("max_k", [100, 300, 1000])
def test_documents_with_more_keys_than_max_k(mz, max_k, nq, dtype):
    """max_k says how the work is cut, not what is read: the same result for any."""
    q, k, v = tensors(nq, 2000, 4, 2, 64, dtype)
    check(mz, q, k, v, table([nq], [2000]), max_k=max_k)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nq,nk", [(1, 8), (33, 33), (90, 90), (1, 300), (129, 2600)])
@pytest.mark.parametrize("size", [1e-28, 1e-31, 1e-33, 1e-35, 1e-36])
def test_small_values_keep_their_digits(mz, size, nq, nk, dtype):
    """Down to where the results themselves are hardly normal numbers: what is lost below
    is half the distance of two subnormal ones, for each term in fp32, for the result in
    bf16. Also with equal scores, whose own rounding hides nothing of the values'."""
    q, k, v = tensors(nq, nk, 2, 2, 64, dtype)
    for queries in (q, q * 0):
        check(mz, queries, k, (v + 3 * v.sign()) * size, table([nq], [nk]),
              floor=nk * 2.0 ** -149 if dtype == "f32" else 2.0 ** -133)


# ---- tokens of no document -------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("q_lens,q_first", [([20, 30], [10, 60]), ([20, 30], None), ([0, 0], None), ([], None),
                                            ([60, 50], [40, 100]), ([100], None)])
def test_tokens_of_no_document_come_back_empty(mz, q_lens, q_first, dtype):
    """0 and -inf, whatever the memory held that the output was made in."""
    import torch
    q, k, v = tensors(100, 160, 2, 2, 64, dtype)
    docs = mz.Documents.of(q_lens, q_first=q_first)
    for _ in range(3):
        torch.full((100, 2, 64), 7.0, dtype=q.dtype, device="cuda")  # (freed at once: the next allocations' memory)
        torch.full((100, 2), 7.0, device="cuda")
        out, lse = mz.attention(q, k, v, docs, return_lse=True)
        bare = torch.ones(100, dtype=torch.bool)
        at = 0
        for i, n in enumerate(q_lens):
            first = q_first[i] if q_first else at
            bare[first:first + n] = False
            at += n
        assert bool((out[bare] == 0).all()) and bool((lse[bare] == -math.inf).all())
        assert bool(torch.isfinite(out[~bare].float()).all()) and bool(torch.isfinite(lse[~bare]).all())
