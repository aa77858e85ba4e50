"""The token loss on the GPU, through the binding, against torch in 64 bits.

Bar: with r the row's maximum, each term's exponent (x - r) log2 e is rounded
twice (2^-23 |x - r| of it), v_exp_f32 and the running sum add at most
2^-23 * (terms of one lane + joins), and the last two steps round values of the
size of max|x| and of the loss. So |error| <= 2^-23 * (V / 256 + 64 + span
+ 2 max|x|) with span = 40, past which a term is below the sum's rounding.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mz():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible GPU"
    from paper_2306_10015_amd import mezo
    return mezo


def reference(x, t):
    import torch
    x = x.double()
    own = x.gather(1, t.clamp(min=0)[:, None])[:, 0]
    losses = torch.where(t >= 0, torch.logsumexp(x, 1) - own, torch.zeros_like(own))
    return losses, losses.sum() / max(1, int((t >= 0).sum()))


def make(rows, vocab, seed, dtype="f32", pad=0, std=3.0, skip=0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty(rows, vocab + pad, device="cuda").normal_(0, std, generator=g)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    if skip:
        t[torch.randperm(rows, generator=g, device="cuda")[:skip]] = -100
    return (x.bfloat16() if dtype == "bf16" else x)[:, :vocab], t


def check(mz, x, t):
    import torch
    losses, mean = mz.token_loss(x, t)
    want, want_mean = reference(x, t)
    tol = 2.0 ** -23 * (x.shape[1] / 256 + 64 + 40 + 2 * x.double().abs().amax(1))
    assert losses.dtype == torch.float32 and losses.shape == (x.shape[0],)
    assert bool(((losses.double() - want).abs() <= tol).all())
    assert abs(float(mean) - float(want_mean)) <= float(tol.max()) + 2.0 ** -23 * abs(float(want_mean))
    return losses, mean


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (1, 2, 0), (5, 3, 2), (3, 63, 1), (7, 64, 0), (2, 65, 7),
                                            (9, 255, 0), (4, 1000, 3), (6, 2047, 1), (3, 2048, 0), (5, 2049, 5),
                                            (2, 4099, 0), (1, 50272, 0), (3, 50272, 8), (17, 50273, 0), (40, 9001, 9),
                                            (300, 5000, 0), (1100, 700, 1), (513, 17000, 3)])
def test_losses_and_mean(mz, rows, vocab, pad, dtype):
    x, t = make(rows, vocab, rows + vocab, dtype, pad, skip=rows // 3)
    check(mz, x, t)


@pytest.mark.parametrize("rows,vocab", [(1, 50272), (4, 9000), (600, 5000), (5, 100)])
def test_large_offsets_and_spread(mz, rows, vocab):
    """Logits far from zero and of a wide spread keep their digits."""
    x, t = make(rows, vocab, 3, std=30.0)
    check(mz, x + 1000.0, t)
    check(mz, x - 5000.0, t)


def test_order_of_rising_and_falling_maxima(mz):
    import torch
    v = 9000
    up = torch.linspace(-80, 80, v, device="cuda")
    x = torch.stack([up, up.flip(0), -up.abs(), up.abs()])
    check(mz, x, torch.tensor([0, 5, v // 2, v - 1], device="cuda"))


@pytest.mark.parametrize("rows,vocab", [(6, 50272), (6, 300), (700, 3000)])
def test_uncounted_rows(mz, rows, vocab):
    """Nothing of an uncounted row is used, NaN included; none counted: 0."""
    import torch
    x, t = make(rows, vocab, 4)
    t[::2] = -1
    x[::2] = float("nan")
    losses, mean = mz.token_loss(x, t)
    want, _ = reference(x[1::2], t[1::2])
    assert bool((losses[::2] == 0).all())
    assert torch.allclose(losses[1::2].double(), want, rtol=0, atol=1e-4)
    assert abs(float(mean) - float(want.mean())) < 1e-4
    losses, mean = mz.token_loss(x, torch.full_like(t, -100))
    assert float(mean) == 0.0 and bool((losses == 0).all())


@pytest.mark.parametrize("rows,vocab", [(8, 50272), (8, 300), (700, 3000)])
def test_special_values(mz, rows, vocab):
    import torch
    x, t = make(rows, vocab, 5)
    inf, nan = float("inf"), float("nan")
    t[:8] = 7
    x[0, 3] = -inf              # a masked word: no part of the sum
    x[1, 7] = -inf              # the target masked: an infinite loss
    x[2] = -inf                 # nothing left
    x[3, 0] = inf
    x[4, vocab - 1] = nan
    t[5] = vocab                # no such word
    t[6] = 1 << 40
    x[7, :] = torch.finfo(torch.float32).min
    losses, mean = mz.token_loss(x, t)
    want, _ = reference(x[:1], t[:1])
    assert abs(float(losses[0]) - float(want)) < 1e-4
    assert float(losses[1]) == inf
    assert all(np.isnan(float(losses[i])) for i in (2, 3, 4, 5, 6)) and np.isnan(float(mean))
    assert abs(float(losses[7]) - np.log(vocab)) < 1e-3 or float(losses[7]) == 0.0  # ln V vanishes next to 3.4e38
    assert bool(torch.isfinite(losses[8:]).all())


def test_equal_inputs_equal_bits(mz):
    import torch
    for rows, vocab in [(1, 50272), (5, 20000), (900, 5000)]:
        x, t = make(rows, vocab, 6)
        a, b = mz.token_loss(x, t), mz.token_loss(x.clone(), t)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_other_stream_and_graph(mz):
    import torch
    for rows, vocab in [(3, 50272), (600, 4000)]:
        x, t = make(rows, vocab, 7)
        want = mz.token_loss(x, t)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        got = mz.token_loss(x, t, stream=s)
        s.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = mz.token_loss(x, t)
        for i in range(3):
            x.copy_(make(rows, vocab, 30 + i)[0])
            eager = mz.token_loss(x, t)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])


def test_refusals(mz):
    import torch
    x, t = make(4, 100, 8)
    with pytest.raises(TypeError):
        mz.token_loss(x, t.int())
    with pytest.raises(TypeError):
        mz.token_loss(x.half(), t)
    with pytest.raises(ValueError):
        mz.token_loss(x, t[:3])
    with pytest.raises(ValueError):
        mz.token_loss(x.t(), t)
    with pytest.raises(ValueError):
        mz.token_loss(x, t.cpu())
    with pytest.raises(ValueError):
        mz.token_loss(x[:0], t[:0])
