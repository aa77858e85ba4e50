"""Every kernel of the product with 4-bit weights on the GPU (nf4_tiles.py), against the
product of the values that the storage holds, in 64 bits.

Bars, from the arithmetic, with u = 2^-24:
- of each element, whatever the order of the sums: bf16 (k + 8) u sum|x w| of exact products, fp32
  (6 k + 8) u sum|x w| of six parts each, and the rounding of the result;
- fp32, of all elements together, sharper: products are within 2^-22 = 4 u of themselves, and of the 6 k
  / 4 additions (a matrix instruction adds at least four products before it rounds) each is off by
  u / sqrt(3) of the sum so far in the mean, which is at most S = sqrt(sum (x w)^2) in the mean: errors have a
  mean square of at most (sqrt(k / 2) + 4 + 1)^2 u^2 S^2, the 1 for the result's rounding. At k = 600 that is
  22 u S; a product that lacked the last 8 of an operand's 24 bits would be off by 40 u S or more;
- fp32, of single products: 2^-22 for the product, u for the sum of its parts and u for a scale or the result."""
import math

import numpy as np
import pytest
import torch

from nf4_tiles import PRODUCTS
from oracle import nf4

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def weights(mz, n, k, absmax, g, code=None):
    """Codes (random ones) of a [n, k] matrix with these scales, and what they stand for in fp32."""
    if code is None:
        code = torch.randint(0, 16, (n * k + 1,), generator=g, device="cuda", dtype=torch.uint8)
    pairs = code[:(n * k + 1) // 2 * 2].view(-1, 2)
    w = mz.NF4Tensor((pairs[:, 0] | pairs[:, 1] << 4).contiguous(), absmax, n * k)
    table = torch.from_numpy(nf4.table().astype(np.float32)).cuda()
    return w, (table[code[:n * k].int()] * absmax.repeat_interleave(64)[:n * k]).view(n, k)


def products(mz, x, w, n, wide, out):
    """Into an array of its own, or into the middle of a wider one."""
    dt = DTYPES[out]
    if not wide:
        return mz.nf4_linear(x, w, dt)
    room = torch.full((x.shape[0], n + 23), 7.0, dtype=dt, device="cuda")
    got = mz.nf4_linear(x, w, dt, out=room[:, 9:9 + n])
    assert bool((room[:, :9] == 7).all()) and bool((room[:, 9 + n:] == 7).all())
    return got


@pytest.mark.parametrize("m,n,k,dtype,kernel,splits,slab,wide", PRODUCTS)
def test_product_of_every_kernel(mz, m, n, k, dtype, kernel, splits, slab, wide):
    g = torch.Generator("cuda").manual_seed(m + n + k)
    # (scales from block to block and rows from one to another by up to 2^4, so that a wrong one shows)
    absmax = 0.02 * torch.exp2(4 * torch.rand((n * k + 63) // 64, generator=g, device="cuda"))
    w, wv = weights(mz, n, k, absmax, g)
    x = torch.randn(m, k, generator=g, device="cuda") * torch.exp2(4 * torch.rand(m, 1, generator=g, device="cuda"))
    x = x.to(DTYPES[dtype])
    xv, wv = x.double(), wv.to(DTYPES[dtype]).double()
    want, sizes = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    steps = k + 8 if dtype == "bf16" else 6 * k + 8
    for out in DTYPES:
        got = products(mz, x, w, n, wide, out).double()
        bar = steps * U * sizes + (U if out == "f32" else 2.0 ** -8) * want.abs()
        assert bool(((got - want).abs() <= bar).all()), (out, float(((got - want).abs() / bar).max()))
        if dtype == out == "f32":
            mean_square = (xv ** 2) @ (wv ** 2).t().contiguous()
            off = float(((got - want) ** 2 / mean_square).mean().sqrt())
            assert off <= (math.sqrt(k / 2) + 5) * U, off / U


@pytest.mark.parametrize("m,n,k,kernel,splits,slab,wide",
                         [p[:3] + p[4:] for p in PRODUCTS if p[3] == "f32" and p[0] * p[1] < 10 ** 7 and p[2] < 10 ** 4])
def test_single_products_of_fp32(mz, m, n, k, kernel, splits, slab, wide):
    """One activation that is not 0 a row: each result is one product of two floats with all their bits."""
    g = torch.Generator("cuda").manual_seed(m + n + k)

    def floats(count):
        """Random ones, and those whose parts after the first are as large as they get."""
        x = 1 + torch.rand(count, generator=g, device="cuda")
        hard = torch.tensor([1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 - 2.0 ** -16 - 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -17,
                             1 + 2.0 ** -7 - 2.0 ** -16 + 2.0 ** -17], device="cuda")
        pick = torch.randint(0, 8, (count,), generator=g, device="cuda")
        x = torch.where(pick < 4, hard[pick.clamp(max=3)], x)
        return x * torch.exp2(torch.randint(-3, 4, (count,), generator=g, device="cuda").float())

    code = torch.randint(0, 16, (n * k + 1,), generator=g, device="cuda", dtype=torch.uint8)
    code = torch.where(torch.rand(n * k + 1, generator=g, device="cuda") < 0.3, torch.full_like(code, 15), code)
    w, wv = weights(mz, n, k, floats((n * k + 63) // 64), g, code)
    at = torch.randint(0, k, (m,), generator=g, device="cuda")
    x = torch.zeros(m, k, device="cuda")
    x[torch.arange(m, device="cuda"), at] = floats(m)
    want = x.sum(1).double()[:, None] * wv.double()[:, at].t()
    off = (products(mz, x, w, n, wide, "f32").double() - want).abs()
    assert bool((off <= (2.0 ** -22 + 2 * U) * want.abs()).all()), float((off / want.abs().clamp(min=1e-30)).max()) / U
