"""Inputs that require a gradient, on the GPU: the operators compute the same, and a
backward pass through them raises instead of leaving their gradient out."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def test_a_loss_in_a_differentiable_model(mz):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(20, 256, generator=g, device="cuda")
    scale = torch.ones(256, device="cuda", requires_grad=True)
    w = mz.f8_quantize(torch.randn(100, 256, generator=g, device="cuda", requires_grad=True))
    t = torch.arange(20, device="cuda")
    docs = mz.Documents.of([20])

    def model(x):
        h = mz.f8_linear(x, w)
        a, lse = mz.attention(x.view(20, 4, 64), x.view(20, 4, 64), x.view(20, 4, 64), docs, return_lse=True)
        return h, a, lse, *mz.token_loss(x, t)

    plain = model(x)
    assert not any(o.requires_grad for o in plain)
    with torch.no_grad():
        assert not any(o.requires_grad for o in model(x * scale))
    for o, p in zip(model(x * scale), plain):
        assert torch.equal(o, p) and o.requires_grad
        with pytest.raises(RuntimeError, match="no backward pass"):
            (o.sum() + scale.sum()).backward()
    assert scale.grad is None
