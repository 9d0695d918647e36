"""The feed-forward block: its step against the same step in 64 bits, and training.

Tolerances.  Every linear layer rounds its operands to 3 bits below the leading one
(relative errors uniform up to 2^-4, 2.7% in the mean square) or to 8-bit codes of a
range, so a product of two is a few percent off in the 2-norm, and the gradients of
the first layer pass four such roundings: 15% is asked for.  The clipped norm is exact
to 1e-5 against the gradients that the block made.
"""
import pytest
import torch

from paper_2010_14298_gb300 import ffn, fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def _data(T, D, seed=3):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    return x, x.float() + 0.3 * torch.randn(T, D, generator=g, device="cuda")


def _reference(block, x, target):
    """The unclipped gradients of the block's parameters and the loss, in 64 bits."""
    p = [t.double().detach().clone().requires_grad_() for t in block.parameters]
    xd = x.double().requires_grad_()
    mean = xd.mean(1, keepdim=True)
    var = ((xd - mean) ** 2).mean(1, keepdim=True)
    y = (xd - mean) * (var + 1e-5) ** -0.5 * p[2] + p[3]
    out = xd + torch.relu(y @ p[0].t()) @ p[1].t()
    loss = ((out - target.double()) ** 2).sum() / (2 * x.shape[0])
    return loss, torch.autograd.grad(loss, p + [xd])


@pytest.mark.parametrize("format", ffn.FORMATS)
@pytest.mark.parametrize("T,D,C", [(512, 256, 512), (300, 144, 400)])
def test_a_step_matches_64_bits(format, T, D, C):
    x, target = _data(T, D)
    block = ffn.FfnBlock(T, D, C, format, max_norm=1e9)
    loss, grads = _reference(block, x, target)
    diff = block.forward(x) - target
    got = float(diff.square().sum() / (2 * T))
    assert abs(got / loss.item() - 1) < 0.05
    dx = block.backward(diff / T)
    assert block.check() == 0
    for g, ref in zip(list(block.grads) + [dx], grads):
        assert (g.double() - ref).norm() <= 0.15 * ref.norm()
    norm = sum(float(g.double().square().sum()) for g in block.grads) ** 0.5
    assert abs(float(block.norm) / norm - 1) < 1e-5


def test_gradients_are_clipped():
    x, target = _data(256, 128)
    block = ffn.FfnBlock(256, 128, 256, "fp8", max_norm=0.01)
    block.step(x, target, 0.1)
    assert float(block.norm) > 0.01
    norm = sum(float(g.double().square().sum()) for g in block.grads) ** 0.5
    assert abs(norm / 0.01 - 1) < 1e-4


@pytest.mark.parametrize("format", ffn.FORMATS)
def test_training_lowers_the_loss(format):
    x, target = _data(512, 128)
    block = ffn.FfnBlock(512, 128, 512, format, max_norm=1.0)
    losses = [float(block.step(x, target, 0.03)) for _ in range(30)]
    assert block.check() == 0
    assert losses[-1] < 0.8 * losses[0]


@pytest.mark.parametrize("format", ffn.FORMATS)
def test_the_same_bits_through_ctypes(format, monkeypatch):
    """Where the extension module cannot be built, the calls are marshalled by ctypes."""
    x, target = _data(300, 128)
    first = ffn.FfnBlock(300, 128, 256, format)
    first.step(x, target, 0.01)
    monkeypatch.setattr(fqt, "_native", fqt._CtypesCalls(fqt.load()))
    second = ffn.FfnBlock(300, 128, 256, format)
    second.step(x, target, 0.01)
    assert second.check() == 0
    assert torch.equal(first.norm, second.norm)
    assert all(torch.equal(a, b) for a, b in zip(first.parameters, second.parameters))


def test_formats_and_widths_that_do_not_exist():
    with pytest.raises(ValueError):
        ffn.FfnBlock(16, 32, 32, "int4")
    with pytest.raises(ValueError):
        ffn.FfnBlock(16, 40, 32, "int8")


def test_command():
    ffn.main(["--tokens", "256", "--width", "128", "--hidden", "256", "--steps", "2"])
