"""The shape of a matrix in 4-bit storage, on the GPU: kept where it is known, so that a product
with activations of another width is refused and not taken of a reshaped matrix."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def test_products_of_another_width_are_refused(mz):
    w = mz.nf4_quantize(torch.randn(48, 128, device="cuda"))
    assert w.shape == (48, 128) and w.numel() == 48 * 128
    assert mz.nf4_linear(torch.randn(3, 128, device="cuda"), w).shape == (3, 48)
    for k in (64, 256, 48, 6144, 1):
        with pytest.raises(ValueError, match="columns"):
            mz.nf4_linear(torch.randn(3, k, device="cuda"), w)


def test_shapes_come_from_the_values(mz):
    values = torch.randn(6, 4, 32, device="cuda")
    w = mz.nf4_quantize(values)
    assert w.shape == (6, 4, 32)
    with pytest.raises(ValueError, match="columns"):
        mz.nf4_linear(torch.randn(2, 32, device="cuda"), w)
    assert mz.nf4_linear(torch.randn(2, 128, device="cuda"), w).shape == (2, 6)  # rows of all that follows the first
    # storage that has a shape keeps it; storage that has none takes the values'
    out = mz.NF4Tensor.empty(24 * 32, shape=(24, 32))
    assert mz.nf4_quantize(values, out) is out and out.shape == (24, 32)
    out = mz.NF4Tensor.empty(24 * 32)
    assert out.shape is None and mz.nf4_quantize(values.view(24, 32), out).shape == (24, 32)


def test_storage_without_a_matrix_takes_the_activations_width(mz):
    w = mz.nf4_quantize(torch.randn(48, 128, device="cuda"))
    flat = mz.NF4Tensor(w.codes, w.absmax, w.numel())
    assert flat.shape is None
    x = torch.randn(3, 128, device="cuda")
    assert torch.equal(mz.nf4_linear(x, flat), mz.nf4_linear(x, w))
    assert mz.nf4_linear(torch.randn(3, 64, device="cuda"), flat).shape == (3, 96)
    line = mz.nf4_quantize(torch.randn(6144, device="cuda"))
    assert line.shape == (6144,) and mz.nf4_linear(x, line).shape == (3, 48)


def test_a_shape_of_other_elements_is_refused(mz):
    w = mz.nf4_quantize(torch.randn(48, 128, device="cuda"))
    for shape in ((48, 127), (128,), ()):
        with pytest.raises(ValueError, match="shape"):
            mz.NF4Tensor(w.codes, w.absmax, w.numel(), shape)
