"""Every kernel of the 8-bit product on the GPU, at sizes that end inside its
tiles and over several words of scales (f8_tiles.py), against the product of the
stored values in 64 bits.

Bars, from the arithmetic: fp32 sums exact terms, k * 2^-23 * sum|x w|; bf16 is
rounded once to 2^-8, and the matrix instruction keeps each of a block's 128 terms
to 2^-15 of the block's largest, which is at most the product of its two maxima.
Scales differ by up to 2^8 from block to block and row to row, so that one taken
from another block or row, or too late, shows."""
import pytest

from f8_tiles import PRODUCTS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def operand(rows, cols, seed, std):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty(rows, cols, device="cuda").normal_(0, std, generator=g)
    blocks = (cols + 127) // 128
    e = torch.randint(-4, 5, (rows, blocks), generator=g, device="cuda").float()
    return x * torch.exp2(e).repeat_interleave(128, 1)[:, :cols]


def stored(m):
    """The values of an 8-bit matrix, in 64 bits, padded to whole blocks."""
    import torch
    blocks = m.codes.shape[1] // 128
    scale = torch.exp2(m.scales[:, :blocks].double() - 127)
    return m.codes.view(torch.float8_e4m3fn).double() * scale.repeat_interleave(128, 1)


@pytest.mark.parametrize("m,n,k,out,tile,splits,wide", PRODUCTS)
def test_product_of_every_kernel(mz, m, n, k, out, tile, splits, wide):
    import torch
    x, w = mz.f8_quantize(operand(m, k, 1, 1.0)), mz.f8_quantize(operand(n, k, 2, 0.02))
    dt = torch.float32 if out == "f32" else torch.bfloat16
    room = torch.full((m, n + 23), 7.0, dtype=dt, device="cuda")
    c = room[:, 9:9 + n] if wide else None
    c = mz.f8_matmul(x, w, dt, out=c)
    if wide:
        assert bool((room[:, :9] == 7).all()) and bool((room[:, 9 + n:] == 7).all())
    xv, wv = stored(x), stored(w)
    exact = xv @ wv.t().contiguous()
    if out == "f32":
        bound = k * 2.0 ** -23 * (xv.abs() @ wv.abs().t().contiguous())
    else:
        tops = [v.abs().unflatten(1, (-1, 128)).amax(2) for v in (xv, wv)]
        bound = 2.0 ** -8 * exact.abs() + (1 + 2.0 ** -8) * 128 * 2.0 ** -15 * (tops[0] @ tops[1].t().contiguous())
    off = (c.double() - exact).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
    assert float(off.norm() / exact.norm()) <= (1e-6 if out == "f32" else 2.0 ** -9 + 1e-4)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [4, 100])
@pytest.mark.parametrize("size", [1e-34, 1e-36, 1e-38, 1e-40])
def test_the_smallest_values(mz, size, m, out):
    """Scales down to the smallest, values down to fp32's subnormal ones. fp32 output takes
    what is below bf16's last bit, 2^-133, to the nearer side."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(m)
    x = mz.f8_quantize(torch.empty(m, 256, device="cuda").normal_(0, 1, generator=g) * size)
    w = mz.f8_quantize(torch.empty(64, 256, device="cuda").normal_(0, 1e20, generator=g))
    c = mz.f8_matmul(x, w, torch.float32 if out == "f32" else torch.bfloat16).double()
    xv, wv = stored(x), stored(w)
    exact = xv @ wv.t().contiguous()
    sums = xv.abs() @ wv.abs().t().contiguous()
    if out == "f32":
        bound = 256 * 2.0 ** -23 * sums + 2.0 ** -134 * wv.abs().sum(1)[None, :]
    else:
        tops = [v.abs().unflatten(1, (-1, 128)).amax(2) for v in (xv, wv)]
        bound = 2.0 ** -8 * exact.abs() + (1 + 2.0 ** -8) * 128 * 2.0 ** -15 * (tops[0] @ tops[1].t().contiguous())
    assert bool(((c - exact).abs() <= bound).all()), float(((c - exact).abs() / bound).max())
