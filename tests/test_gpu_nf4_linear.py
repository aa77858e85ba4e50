"""Products with 4-bit weights on the GPU, through the binding, against a plain
product in 64 bits of the values that the storage holds. The bars come from the
arithmetic (bound)."""
import math

import numpy as np
import pytest
import torch

from oracle import nf4

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def weights(mz, n, k, seed=0, scale=0.02):
    """Random codes and scales of a [n, k] matrix, and the codes one by one."""
    g = torch.Generator().manual_seed(seed + 31 * n + k)
    code = torch.randint(0, 16, (n * k,), generator=g)
    packed = torch.zeros((n * k + 1) // 2, dtype=torch.uint8)
    packed |= code[0::2].to(torch.uint8)
    packed[:n * k // 2] |= (code[1::2] << 4).to(torch.uint8)
    absmax = torch.rand((n * k + 63) // 64, generator=g) * scale + scale / 4
    return mz.NF4Tensor(packed.cuda(), absmax.cuda(), n * k), code, absmax


def values(code, absmax, n, k, dtype):
    """What the storage holds, in dtype, as 64-bit numbers (the product of two floats is exact there)."""
    w = torch.from_numpy(nf4.table().astype(np.float64))[code] * absmax.double().repeat_interleave(64)[:n * k]
    return w.float().to(dtype).double().view(n, k)


def bound(x, w, want, out_dtype):
    """bf16: exact products, k of them summed in fp32 in any order, and the result's rounding."""
    return (x.shape[1] + 8) * 2.0 ** -24 * (x.abs() @ w.abs().t()) + rounding(out_dtype) * want.abs() + 1e-37


def bound_f32(x, w, want, out_dtype):
    """fp32: six partial products each, those left out below 2^-23 of the product."""
    return (6 * x.shape[1] + 8) * 2.0 ** -24 * (x.abs() @ w.abs().t()) + rounding(out_dtype) * want.abs() + 1e-37


def rounding(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


def activations(m, k, dtype, pad=0, seed=0):
    g = torch.Generator().manual_seed(seed + 7 * m + k)
    x = torch.randn(m, k + pad, generator=g)
    x[:, :max(1, k // 200)] *= 20
    return x.to(DTYPES[dtype]).cuda()[:, :k]


def check(mz, m, n, k, dtype="bf16", out="bf16", pad=0, **kw):
    w, code, absmax = weights(mz, n, k)
    x = activations(m, k, dtype, pad)
    got = mz.nf4_linear(x, w, None if out == dtype else DTYPES[out], **kw)
    assert got.shape == (m, n) and got.dtype == DTYPES[out]
    wv, xv = values(code, absmax, n, k, DTYPES[dtype]), x.cpu().double()
    want = xv @ wv.t()
    off, bar = (got.cpu().double() - want).abs(), (bound if dtype == "bf16" else bound_f32)(xv, wv, want, DTYPES[out])
    assert bool((off <= bar).all()), float((off / bar).max())
    return got


FORMS = [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("dtype,out", FORMS)
@pytest.mark.parametrize("m", [1, 2, 3, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 129, 200, 257])
def test_rows(mz, m, dtype, out):
    check(mz, m, 192, 256, dtype, out)


@pytest.mark.parametrize("dtype,out", FORMS)
@pytest.mark.parametrize("n", [1, 3, 15, 16, 17, 63, 64, 65, 127, 130, 300])
@pytest.mark.parametrize("m", [1, 20, 70])
def test_columns(mz, n, m, dtype, out):
    check(mz, m, n, 320, dtype, out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [1, 2, 7, 8, 31, 32, 33, 63, 64, 65, 127, 128, 192, 200, 255, 256, 320, 448, 512, 513, 576,
                               960, 1000, 1024, 2050, 4160])
@pytest.mark.parametrize("m", [1, 24, 80])
def test_lengths_of_the_sum(mz, k, m, dtype):
    """Blocks that run over the ends of rows, rows that begin within a byte, and every last stage."""
    check(mz, m, 70, k, dtype, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [1, 3, 4, 8, 64])
@pytest.mark.parametrize("m", [1, 5, 90])
def test_rows_apart(mz, pad, m, dtype):
    check(mz, m, 100, 256, dtype, dtype, pad=pad)
    w, _, _ = weights(mz, 100, 256)
    x = activations(m, 256, dtype)
    want = mz.nf4_linear(x, w)
    shifted = torch.zeros(m, 256 + pad, dtype=x.dtype, device="cuda")
    shifted[:, pad:] = x  # (rows begin at any element)
    assert torch.equal(mz.nf4_linear(shifted[:, pad:], w), want)
    wide = torch.full((m, 100 + pad), 7.0, dtype=x.dtype, device="cuda")
    assert torch.equal(mz.nf4_linear(x, w, out=wide[:, pad:]), want)
    assert bool((wide[:, :pad] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(1, 768, 768), (1, 2048, 8192), (24, 768, 4096), (64, 50, 16384), (300, 1000, 1024),
                                   (700, 520, 640), (513, 2100, 512), (2000, 777, 448), (1, 50001, 192), (4, 50001, 64),
                                   (30, 50001, 128)])
def test_larger_products(mz, m, n, k, dtype):
    check(mz, m, n, k, dtype, dtype)


def test_values_are_those_of_the_conversion(mz):
    """One row of the identity at a time: each weight comes out as nf4_dequantize gives it."""
    for dtype in DTYPES.values():
        for n, k in ((40, 128), (17, 100)):
            w, _, _ = weights(mz, n, k)
            eye = torch.eye(k, dtype=dtype, device="cuda")
            want = mz.nf4_dequantize(w, dtype).view(n, k)
            assert torch.equal(mz.nf4_linear(eye, w).t(), want)
            assert torch.equal(mz.nf4_linear(eye[:9], w).t(), want[:, :9])
            assert torch.equal(mz.nf4_linear(eye[3:4], w).t(), want[:, 3:4])


def test_quantized_weights(mz):
    w = torch.randn(100, 192, device="cuda", generator=torch.Generator("cuda").manual_seed(0)) * 0.05
    x = activations(30, 192, "bf16")
    q = mz.nf4_quantize(w)
    want = x.cpu().double() @ mz.nf4_dequantize(q, torch.bfloat16).view(100, 192).cpu().double().t()
    got = mz.nf4_linear(x, q, torch.float32).cpu().double()
    wv = mz.nf4_dequantize(q, torch.bfloat16).view(100, 192).cpu().double()
    assert bool(((got - want).abs() <= bound(x.cpu().double(), wv, want, torch.float32)).all())


@pytest.mark.parametrize("m", [1, 40, 100])
@pytest.mark.parametrize("power", [-100, -60, 60, 100])
def test_the_range_of_fp32(mz, power, m):
    """Activations and scales far from 1, their products within the range."""
    w, code, absmax = weights(mz, 33, 128)
    w.absmax.mul_(2.0 ** -power)
    absmax = absmax * 2.0 ** -power
    x = activations(m, 128, "f32") * 2.0 ** power
    got = mz.nf4_linear(x, w).cpu().double()
    wv, xv = values(code, absmax, 33, 128, torch.float32), x.cpu().double()
    want = xv @ wv.t()
    assert bool(((got - want).abs() <= bound_f32(xv, wv, want, torch.float32)).all())


@pytest.mark.parametrize("m", [1, 20, 100])
def test_the_largest_floats(mz, m):
    """Values that rounding to bf16 would make infinite stay finite."""
    w, code, absmax = weights(mz, 20, 64, scale=1e-3)
    x = torch.zeros(m, 64, device="cuda")
    x[:, 5] = 3.4028234e38
    got = mz.nf4_linear(x, w).cpu().double()
    wv = values(code, absmax, 20, 64, torch.float32)
    want = x.cpu().double() @ wv.t()
    assert bool(((got - want).abs() <= bound_f32(x.cpu().double(), wv, want, torch.float32)).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("m", [1, 20, 100])
def test_values_that_are_not_finite(mz, m, bad, dtype):
    """They stay in their row of x, and in the outputs of their block."""
    w, _, _ = weights(mz, 70, 128)
    x = activations(m, 128, dtype)
    want = mz.nf4_linear(x, w)
    y = x.clone()
    y[m - 1, 77] = bad
    got = mz.nf4_linear(y, w)
    assert torch.equal(got[:m - 1], want[:m - 1])
    zero = mz.nf4_dequantize(w).view(70, 128)[:, 77] == 0
    assert not bool(torch.isfinite(got[m - 1][~zero].float()).any())
    if bad != bad:
        assert bool(torch.isnan(got[m - 1].float()).all())
    low = torch.full((1,), 0x7F800001, dtype=torch.int32).view(torch.float32).cuda()  # a NaN in its last bit
    if dtype == "f32":
        y[m - 1, 77] = low[0]
        y.view(torch.int32)[m - 1, 77] = 0x7F800001
        assert bool(torch.isnan(mz.nf4_linear(y, w)[m - 1]).all())
    w.absmax[2 * 9 + 1] = bad  # row 9, columns 64 .. 127
    got = mz.nf4_linear(x, w)
    rest = [i for i in range(70) if i != 9]
    assert torch.equal(got[:, rest], want[:, rest]) and not bool(torch.isfinite(got[:, 9].float()).any())


def test_scales_of_zero(mz):
    w, _, _ = weights(mz, 64, 64)
    w.absmax.zero_()
    for m in (1, 30, 100):
        assert bool((mz.nf4_linear(activations(m, 64, "bf16"), w) == 0).all())


def test_equal_inputs_give_equal_bits(mz):
    for m, n, k in ((1, 768, 768), (24, 200, 8192), (128, 300, 4096), (600, 600, 1024)):
        for dtype in DTYPES:
            w, _, _ = weights(mz, n, k)
            x = activations(m, k, dtype)
            first = mz.nf4_linear(x, w)
            assert all(torch.equal(mz.nf4_linear(x, w), first) for _ in range(3))


def test_what_lies_behind_the_last_row_is_left_alone(mz):
    for m, n, k in ((1, 65, 128), (30, 65, 128), (100, 65, 128), (3, 65, 100)):
        for dtype in DTYPES.values():
            w, _, _ = weights(mz, n, k)
            room = torch.full((m * n + 64,), 7.0, dtype=dtype, device="cuda")
            mz.nf4_linear(activations(m, k, "bf16").to(dtype), w, out=room[:m * n].view(m, n))
            assert bool((room[m * n:] == 7).all())


def test_slabs_of_a_large_matrix(mz):
    """More expanded weights than are kept at a time: every slab with its own rows."""
    n, k, m = 5000, 23000, 70
    for dtype in DTYPES:
        w, code, absmax = weights(mz, n, k)
        x = activations(m, k, dtype)
        got = mz.nf4_linear(x, w, torch.float32)
        dense = mz.nf4_dequantize(w, DTYPES[dtype]).view(n, k)
        for rows in (slice(0, 40), slice(1800, 1900), slice(n - 40, n)):
            want = x.double() @ dense[rows].double().t().contiguous()
            size = x.double().abs() @ dense[rows].double().abs().t().contiguous()
            assert bool(((got[:, rows].double() - want).abs() <= (6 * k + 8) * 2.0 ** -24 * size).all())
        # one slab's rows alone give the same
        part = mz.nf4_linear(x, mz.NF4Tensor(w.codes[:64 * k // 2], w.absmax[:64 * k // 64 + 1], 64 * k), torch.float32)
        assert float((part - got[:, :64]).abs().max()) <= float((6 * k + 8) * 2.0 ** -23 * size.max())


def test_refusals(mz):
    w, _, _ = weights(mz, 10, 64)
    x = activations(4, 64, "bf16")
    for bad in (lambda: mz.nf4_linear(x[:, :60], w), lambda: mz.nf4_linear(x.t(), w), lambda: mz.nf4_linear(x[0], w),
                lambda: mz.nf4_linear(x[:0], w), lambda: mz.nf4_linear(x.cpu(), w),
                lambda: mz.nf4_linear(x, w, out=torch.empty(4, 9, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: mz.nf4_linear(x.half(), w), lambda: mz.nf4_linear(x, w, torch.float16),
                lambda: mz.nf4_linear(x, w, torch.float32, out=torch.empty(4, 10, device="cuda").bfloat16())):
        with pytest.raises(TypeError):
            bad()


def test_another_stream_and_a_graph(mz):
    for m, dtype in ((1, "bf16"), (100, "f32"), (1, "f32")):
        w, _, _ = weights(mz, 300, 1024)
        x = activations(m, 1024, dtype)
        want = mz.nf4_linear(x, w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = mz.nf4_linear(x, w, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
        y, out = x.clone(), torch.empty_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mz.nf4_linear(y, w, out=out)
        for step in range(3):
            y.copy_(x * (step + 1))
            graph.replay()
            replayed = out.clone()
            torch.cuda.synchronize()
            assert torch.equal(replayed, mz.nf4_linear(y, w))


def test_no_backward(mz):
    w, _, _ = weights(mz, 10, 64)
    x = activations(4, 64, "f32").clone().requires_grad_(True)
    with pytest.raises(RuntimeError, match="no backward pass"):
        mz.nf4_linear(x, w).sum().backward()
    assert np.isfinite(float(mz.nf4_linear(x.detach(), w).sum()))


@pytest.mark.parametrize("dtype,out", FORMS)
@pytest.mark.parametrize("m", [1, 5, 16, 17, 32, 33, 64, 65])
@pytest.mark.parametrize("n,k", [(33, 100), (4097, 77), (5000, 30), (100, 5001)])
def test_rows_that_end_within_a_block(mz, n, k, m, dtype, out):
    check(mz, m, n, k, dtype, out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [50, 100, 131])
def test_blocks_that_are_not_finite_reach_their_own_rows(mz, k, dtype):
    """A block of the next row alone changes nothing, though it is read with the last columns."""
    n, m = 40, 3
    w, code, absmax = weights(mz, n, k)
    x = activations(m, k, dtype)
    want = mz.nf4_linear(x, w)
    for b in (1, 17, absmax.numel() - 1):
        own = torch.zeros(n, dtype=torch.bool)
        own[b * 64 // k:min(n, (min(b * 64 + 63, n * k - 1)) // k + 1)] = True
        for bad in (math.nan, math.inf):
            w.absmax[b] = bad
            got = mz.nf4_linear(x, w).cpu()
            assert torch.equal(got[:, ~own], want.cpu()[:, ~own])
            assert not bool(torch.isfinite(got[:, own]).any())
        w.absmax[b] = absmax[b]
