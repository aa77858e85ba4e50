"""The forward-only example (examples/forward_only.py): the engine and the
forward pass's operators together, as a user's program runs them."""
import os
import sys

import pytest

import attention_ref
import f8_ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module")
def example():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    import forward_only
    return forward_only


def plain_loss(model, words, targets, docs):
    """The model's loss with every operator replaced by its reference in 64
    bits; activations rounded to bf16 where the model keeps them so."""
    import torch

    def linear(x, w):
        xv = f8_ref.dequantize(*f8_ref.quantize(x.float().numpy()), x.shape[1])
        wv = f8_ref.dequantize(*f8_ref.quantize(w.float().cpu().numpy()), w.shape[1])
        return torch.from_numpy(xv @ wv.T)

    rows = [tuple(r) for r in docs.table.tolist()]
    h, hk, d, width = model.heads, model.kv_heads, model.dim, model.width
    norm = torch.nn.functional.rms_norm
    x = model.weights[0].cpu()[words.cpu()]
    for i in range(1, len(model.weights), 4):
        qkv_w, out_w, up_w, down_w = model.weights[i:i + 4]
        qkv = linear(norm(x, (width,)), qkv_w).bfloat16().view(-1, h + 2 * hk, d)
        a, _, _ = attention_ref.attention(qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:], rows, slopes=model.slopes.cpu())
        x = x + linear(a.bfloat16().flatten(1), out_w).bfloat16()
        x = x + linear(torch.relu(linear(norm(x, (width,)), up_w).bfloat16()), down_w).bfloat16()
    logits, t = linear(norm(x, (width,)), model.weights[0]), targets.cpu()
    losses = torch.logsumexp(logits, 1) - logits.gather(1, t.clamp(min=0)[:, None])[:, 0]
    return float(losses[t >= 0].mean())


def test_loss_against_the_plain_model(example):
    """Operators and reference round at the same places; a sum that falls on the
    other side of a rounding moves an activation by 2^-8 of itself, of which the
    loss, a mean over 20 tokens of values near 3, keeps less than 1 in 100."""
    model = example.Decoder(vocab=40, seed=3)
    data = example.batch(40, 20, 7)
    got = float(model.loss(*data))
    assert abs(got - plain_loss(model, *data)) <= 0.03


def test_runs_repeat_bit_for_bit(example):
    """The same seeds give the same losses, and so the same weights, every time."""
    a = example.train(steps=12, samples=3, count=16, seed=1)
    b = example.train(steps=12, samples=3, count=16, seed=1)
    assert a == b and all(x == x and abs(x) < 100 for x in a)


def test_it_learns(example):
    """From a loss of about 5 to below the ln 2 of one who only knows the two
    names: the halves are told apart."""
    history = example.train(steps=200, samples=16)
    assert sum(history[-20:]) / 20 < 0.69 < sum(history[:5]) / 5
