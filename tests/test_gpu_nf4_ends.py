"""fp32 products with 4-bit weights at the ends of the range, on the GPU, by every kind of kernel:
few activations, rows of weights that end within a block, and tiles. Bars as in
test_gpu_nf4_tiles.py: of a single product 2^-22, and u = 2^-24 for the sum of its parts and for a
scale or the result."""
import math

import numpy as np
import pytest
import torch

from oracle import nf4

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LARGEST = float(np.finfo(np.float32).max)
# (m, n, k): few activations, ragged rows, tiles of ragged and of whole rows
SIZES = [(20, 70, 128), (10, 70, 100), (100, 70, 100), (1100, 70, 128)]


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def weights(mz, n, k, absmax):
    g = torch.Generator("cuda").manual_seed(n + k)
    code = torch.randint(0, 16, (n * k,), generator=g, device="cuda", dtype=torch.uint8)
    absmax = absmax if torch.is_tensor(absmax) else torch.full(((n * k + 63) // 64,), absmax, device="cuda")
    w = mz.NF4Tensor((code[0::2] | code[1::2] << 4).contiguous(), absmax, n * k)
    table = torch.from_numpy(nf4.table().astype(np.float32)).cuda()
    return w, (table[code.int()] * absmax.repeat_interleave(64)[:n * k]).view(n, k)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("activations", [True, False])
def test_the_largest_floats(mz, activations, m, n, k):
    """Those that rounding to bf16 would make infinite too."""
    large = torch.tensor([LARGEST, -LARGEST] + [(-1) ** i * float.fromhex(x) for i, x in enumerate(
        ("0x1.FEp127", "0x1.FFp127", "0x1.FEFFFEp127", "0x1.FF0002p127"))], device="cuda")
    g = torch.Generator("cuda").manual_seed(m)
    at = torch.randint(0, k, (m,), generator=g, device="cuda")
    x = torch.zeros(m, k, device="cuda")
    if activations:
        w, wv = weights(mz, n, k, 0.7)
        x[torch.arange(m, device="cuda"), at] = large[torch.arange(m, device="cuda") % 6]
    else:
        w, wv = weights(mz, n, k, large.abs()[torch.arange((n * k + 63) // 64, device="cuda") % 6])
        x[torch.arange(m, device="cuda"), at] = 0.5 + torch.rand(m, generator=g, device="cuda") / 2
    want = x.sum(1).double()[:, None] * wv.double()[:, at].t()
    off = (mz.nf4_linear(x, w).double() - want).abs()
    assert bool((off <= (2.0 ** -22 + 2 * U) * want.abs()).all())


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("bits", [0x7F800000, 0xFF800000, 0x7FC00000, 0x7F800001, 0xFF80FFFF])
def test_values_that_are_not_finite(mz, bits, m, n, k):
    """Infinities and NaN, those by their low bits alone among them, stay in their row of x, and in the rows of
    weights that their block is of."""
    g = torch.Generator("cuda").manual_seed(m + k)
    x = torch.randn(m, k, generator=g, device="cuda")
    w, wv = weights(mz, n, k, 0.3)
    want = mz.nf4_linear(x, w)
    bad = torch.tensor([bits if bits < 2 ** 31 else bits - 2 ** 32], dtype=torch.int32, device="cuda")
    y = x.clone()
    y.view(torch.int32)[m - 1, k - 1] = bad[0]
    got = mz.nf4_linear(y, w)
    assert torch.equal(got[:m - 1], want[:m - 1])
    nonzero = wv[:, k - 1] != 0
    assert not bool(torch.isfinite(got[m - 1][nonzero]).any())
    b = (n // 2 * k + k // 2) // 64
    w.absmax.view(torch.int32)[b] = bad[0]
    got = mz.nf4_linear(x, w)
    own = torch.zeros(n, dtype=torch.bool, device="cuda")
    own[b * 64 // k:(b * 64 + 63) // k + 1] = True
    assert torch.equal(got[:, ~own], want[:, ~own]) and not bool(torch.isfinite(got[:, own]).any())


def test_sums_that_end_in_range(mz):
    """Terms near the largest float of either sign, their sum small: no step of the way is infinite."""
    for m, n, k in SIZES:
        w, wv = weights(mz, n, k, 1.0)
        x = torch.zeros(m, k, device="cuda")
        x[:, 3], x[:, k - 2] = LARGEST / 4, -LARGEST / 4
        got = mz.nf4_linear(x, w)
        want = x.double() @ wv.double().t()
        size = x.double().abs() @ wv.double().abs().t()
        assert bool(torch.isfinite(got).all()) and math.isfinite(float(size.max()))
        assert bool(((got.double() - want).abs() <= (2.0 ** -22 + 12 * U) * size).all())
