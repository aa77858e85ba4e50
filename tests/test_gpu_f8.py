"""8-bit storage and its product on the GPU, through the binding, against a
plain reference in 64 bits (f8_ref.py).

Bars, all from the arithmetic:
  codes and scales are bit-exact (a power of two scales exactly, a code is one
  rounding); fp32 products are sums of exact terms in fp32: within
  k * 2^-23 * sum|x w| of the exact sum; bf16 products: one rounding of 2^-8 (8 significant bits),
  and the matrix instruction's inner sum, which keeps each of a block's 128
  terms to 2^-15 of the block's largest.
"""
import numpy as np
import pytest

import f8_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def values(rows, cols, seed, std=0.02):
    return np.random.Generator(np.random.PCG64([seed, rows, cols])).normal(0, std, (rows, cols)).astype(np.float32)


def host(m):
    return m.codes.cpu().numpy(), m.scales.cpu().numpy()


def same_codes(got, want):
    """Bytes equal, except that NaN may have either sign."""
    nan = (want & 127) == 127
    return np.array_equal(got[~nan], want[~nan]) and bool(np.all((got[nan] & 127) == 127))


def check_quantized(mz, dev, w):
    q = mz.f8_quantize(dev)
    codes, scales = f8_ref.quantize(w)
    got_c, got_s = host(q)
    assert np.array_equal(got_s, scales)
    assert same_codes(got_c, codes)
    return q


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 128), (5, 129), (17, 500), (4, 513), (33, 768), (1, 2050)])
def test_quantize_bit_exact(mz, rows, cols, dtype):
    import torch
    w = torch.from_numpy(values(rows, cols, 1))
    if dtype == "bf16":
        w = w.bfloat16()
    check_quantized(mz, w.cuda(), w.float().numpy())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 3), (8, 8), (5, 0), (4, 24)])
def test_quantize_rows_of_a_wider_array(mz, offset, pad, dtype):
    """Any row stride and any first column, aligned for wide loads or not."""
    import torch
    w = torch.from_numpy(values(9, 300 + offset + pad, 2))
    if dtype == "bf16":
        w = w.bfloat16()
    check_quantized(mz, w.cuda()[:, offset:offset + 300], w[:, offset:offset + 300].float().numpy())


def test_quantize_extremes(mz):
    """Blocks of zeros, of subnormals, of the largest floats, of one value at
    and next to 448 * 2^e, ties, infinities and NaN."""
    import torch
    w = values(12, 384, 3)
    w[0] = 0.0
    w[1, :128] = np.float32(1e-40)
    w[1, 128:256] = np.float32(-1e-45)
    w[2] *= np.float32(1e37)
    w[3, 5] = np.float32(3.4e38)
    w[4] = 0.0
    w[4, 0], w[4, 128], w[4, 256] = 448.0, np.nextafter(np.float32(448.0), np.float32(500)), 449.0
    w[5, :128] = np.float32(448.0) * (np.arange(128, dtype=np.float32) + 0.5) / 128
    w[5, 128:256] = (np.arange(128, dtype=np.float32) * 2 + 1) * np.float32(2.0 ** -10)  # halfway between codes
    w[5, 128] = 448.0
    w[6, 7], w[6, 200], w[6, 300] = np.inf, -np.inf, np.nan
    w[7, :128] = np.nan
    w[8] = -0.0
    w[9, :128] *= np.float32(1e-36)
    w[10, :128] = np.float32(2.0 ** -126)
    check_quantized(mz, torch.from_numpy(w).cuda(), w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_every_exponent(mz, dtype):
    """Rows whose largest exponent field runs from subnormal to the top, with
    elements down to 2^-20 of it and, in bf16, every tie between two codes."""
    import torch
    rng = np.random.Generator(np.random.PCG64(11))
    top = np.arange(255)[:, None]
    exponent = np.maximum(top - rng.integers(0, 20, (255, 512)), 0)
    bits = (rng.integers(0, 2, (255, 512)) << 31 | exponent << 23 | rng.integers(0, 1 << 23, (255, 512)))
    if dtype == "bf16":
        bits &= 0xFFFF0000
    w = bits.astype(np.uint32).view(np.float32)
    dev = torch.from_numpy(w).cuda()
    check_quantized(mz, dev.bfloat16() if dtype == "bf16" else dev, w)


def test_quantize_into_writes_the_padding(mz):
    import torch
    w = torch.from_numpy(values(6, 130, 4))
    out = mz.F8Matrix.empty(6, 130)
    out.codes.fill_(0x55)
    out.scales.fill_(0x55)
    mz.f8_quantize(w.cuda(), out=out)
    codes, scales = f8_ref.quantize(w.numpy())
    assert np.array_equal(out.codes.cpu().numpy(), codes)
    assert np.array_equal(out.scales.cpu().numpy(), scales)


def check_product(mz, x, w, out_dtype, out=None):
    import torch
    xq, wq = mz.f8_quantize(x), mz.f8_quantize(w)
    xv = f8_ref.dequantize(*host(xq), xq.cols)
    wv = f8_ref.dequantize(*host(wq), wq.cols)
    got = mz.f8_matmul(xq, wq, out_dtype, out)
    assert got.shape == (x.shape[0], w.shape[0]) and got.dtype == out_dtype
    g = got.double().cpu().numpy()
    exact = xv @ wv.T
    if out_dtype == torch.float32:
        bound = xv.shape[1] * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T)
    else:
        bound = 2.0 ** -8 * np.abs(exact)
        for b in range(0, xv.shape[1], f8_ref.BLOCK):  # 128 terms, each to 2^-15 of the largest
            xb, wb = np.abs(xv[:, b:b + 128]), np.abs(wv[:, b:b + 128])
            largest = np.stack([(xb * row).max(axis=1) for row in wb], axis=1)
            bound = bound + (1 + 2.0 ** -8) * 128 * 2.0 ** -15 * largest
    assert np.all(np.abs(g - exact) <= bound + 1e-38), float(np.max(np.abs(g - exact) / (bound + 1e-38)))
    norm = np.linalg.norm(g - exact) / np.linalg.norm(exact)
    assert norm <= (1e-6 if out_dtype == torch.float32 else 2.0 ** -9 + 1e-4)
    return got


SIZES = [(1, 1, 1), (1, 768, 768), (2, 50, 130), (3, 17, 128), (16, 64, 512), (17, 130, 640), (33, 100, 1030),
         (64, 257, 300), (65, 64, 256), (100, 200, 129), (129, 300, 900), (300, 129, 64), (257, 520, 384),
         (70, 33, 5000)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product(mz, m, n, k, out):
    import torch
    x = torch.from_numpy(values(m, k, 5, 1.0)).cuda()
    w = torch.from_numpy(values(n, k, 6)).cuda()
    check_product(mz, x, w, torch.float32 if out == "f32" else torch.bfloat16)


@pytest.mark.parametrize("m,n,k", [(1, 1000, 4096), (40, 3000, 2048), (2000, 2100, 512), (4200, 4100, 256)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product_of_small_integers_is_exact(mz, m, n, k, out):
    """Every tile of larger products: integers whose sums every step holds."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n)
    # scales 2^e of blocks in which 448 stands once, against a zero of the other operand
    x = torch.randint(-1, 2, (m, k), generator=g, device="cuda").float()
    w = torch.randint(-1, 2, (n, k), generator=g, device="cuda").float()
    if out == "bf16":  # at most 256 terms that are not zero
        x[:, 256:] = 0
    got = mz.f8_linear(x, mz.f8_quantize(w), torch.float32 if out == "f32" else torch.bfloat16)
    assert torch.equal(got.float(), x @ w.t())


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [5, 90])
def test_scales_of_every_block_and_row(mz, m, out):
    """Rows and blocks of very different sizes: each keeps its own scale."""
    import torch
    r = np.random.Generator(np.random.PCG64(9))
    k = 128 * 9 + 40
    x, w = values(m, k, 7, 1.0), values(75, k, 8, 1.0)
    for v in (x, w):
        for b in range(0, k, 128):
            v[:, b:b + 128] *= np.exp2(r.integers(-20, 20, (v.shape[0], 1))).astype(np.float32)
    check_product(mz, torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda(),
                  torch.float32 if out == "f32" else torch.bfloat16)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [6, 140])
def test_out_may_be_a_part_of_a_wider_array(mz, m, out):
    import torch
    dt = torch.float32 if out == "f32" else torch.bfloat16
    x = torch.from_numpy(values(m, 256, 10, 1.0)).cuda()
    w = torch.from_numpy(values(37, 256, 11)).cuda()
    wide = torch.full((m, 60), 7.0, dtype=dt, device="cuda")
    check_product(mz, x, w, dt, out=wide[:, 9:46])
    assert bool((wide[:, :9] == 7).all()) and bool((wide[:, 46:] == 7).all())


@pytest.mark.parametrize("m", [3, 80])
def test_nan_stays_in_its_row_and_column(mz, m):
    import torch
    x = torch.from_numpy(values(m, 300, 12, 1.0)).cuda()
    w = torch.from_numpy(values(50, 300, 13)).cuda()
    x[1, 5] = float("nan")
    w[7, 290] = float("inf")
    for dt in (torch.float32, torch.bfloat16):
        bad = ~torch.isfinite(mz.f8_linear(x, mz.f8_quantize(w), dt))
        want = torch.zeros_like(bad)
        want[1] = True
        want[:, 7] = True
        assert torch.equal(bad, want)


def test_tiny_scales(mz):
    """Scales down to 2^-127: products of the smallest blocks with large ones."""
    import torch
    x = np.full((2, 128), 1e-37, dtype=np.float32)
    x[1] = 3e-38
    w = np.full((3, 128), 1e30, dtype=np.float32)
    check_product(mz, torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda(), torch.float32)


def test_other_stream_and_graph(mz):
    import torch
    x = torch.from_numpy(values(40, 640, 14, 1.0)).cuda()
    w = mz.f8_quantize(torch.from_numpy(values(90, 640, 15)).cuda())
    want = mz.f8_linear(x, w, torch.bfloat16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = mz.f8_linear(x, w, torch.bfloat16, stream=s)
    raw = mz.f8_linear(x, w, torch.bfloat16, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(raw, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mz.f8_linear(x, w, torch.bfloat16)
    for i in range(3):
        x.copy_(torch.from_numpy(values(40, 640, 20 + i, 1.0)))
        eager = mz.f8_linear(x, w, torch.bfloat16)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_refusals(mz):
    import torch
    x = torch.zeros(4, 256, device="cuda")
    with pytest.raises(TypeError):
        mz.f8_quantize(x.half())
    with pytest.raises(ValueError):
        mz.f8_quantize(x.t()[:, :3])
    with pytest.raises(ValueError):
        mz.f8_quantize(x.cpu())
    with pytest.raises(ValueError):
        mz.f8_quantize(torch.zeros(0, 8, device="cuda"))
    with pytest.raises(ValueError):
        mz.f8_quantize(x, out=mz.F8Matrix.empty(4, 255))
    w = mz.f8_quantize(torch.zeros(8, 128, device="cuda"))
    with pytest.raises(ValueError):
        mz.f8_matmul(mz.f8_quantize(x), w)
    xq = mz.f8_quantize(torch.zeros(4, 128, device="cuda"))
    with pytest.raises(ValueError):
        mz.f8_matmul(xq, w, out=torch.zeros(4, 9, device="cuda"))
    with pytest.raises(TypeError):
        mz.f8_matmul(xq, w, torch.float32, out=torch.zeros(4, 8, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        mz.f8_matmul(xq, w, torch.float16)
    with pytest.raises(ValueError):
        mz.f8_matmul(xq, w, out=torch.zeros(8, 4, device="cuda").t())
    with pytest.raises(mz.MezoError) as e:  # the output over an operand
        mz.f8_matmul(xq, w, out=w.codes.view(torch.float32)[:4, :8])
    assert e.value.code == mz.EOVERLAP
    with pytest.raises(ValueError):
        mz.F8Matrix(w.codes, w.scales, 8, 129)
    with pytest.raises(TypeError):
        mz.F8Matrix(w.codes.view(torch.int8), w.scales, 8, 128)
