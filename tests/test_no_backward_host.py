"""The operators of the forward pass in autograd's graph, on the host: outputs of
inputs that require a gradient lead back to an error, all others to nothing."""
import pytest
import torch

from paper_2306_10015_amd import mezo


def test_backward_through_an_operator_raises():
    x, y = torch.ones(3, requires_grad=True), torch.ones(3)
    out, lse = x.detach() * 2, torch.zeros(2)
    same = out
    mezo._no_backward("attention", (out, lse), x, y, None)
    assert out is same and out.requires_grad and lse.requires_grad
    with pytest.raises(RuntimeError, match="mezo.attention has no backward pass"):
        (out.sum() + x.sum()).backward()
    with pytest.raises(RuntimeError, match="no backward pass"):
        lse.sum().backward()


def test_outputs_of_plain_inputs_stay_plain():
    x, w = torch.ones(3), torch.ones(3, requires_grad=True)
    out = torch.zeros(3)
    mezo._no_backward("f8_linear", (out,), x, None)
    with torch.no_grad():
        mezo._no_backward("f8_linear", (out,), w)
    mezo._no_backward("f8_linear", (out,), w.detach())
    assert not out.requires_grad and out.grad_fn is None


def test_a_part_of_a_wider_array_may_be_the_output():
    w, wide = torch.ones(3, requires_grad=True), torch.zeros(2, 5)
    out = wide[:, 1:4]
    mezo._no_backward("f8_linear", (out,), w)
    with pytest.raises(RuntimeError, match="no backward pass"):
        wide.sum().backward()
