"""The gated feed-forward block: its step against the same step in 64 bits.

Tolerances.  As for the block without a gate: an operand's rounding to 3 bits below the
leading one is 2.7% of it in the mean square, and a gradient passes at most eight of them:
15% in the 2-norm.  (relu's slope jumps, which its own test of a step allows for; the smooth
activations are taken here.)  The clipped norm is exact to 1e-5 against the gradients that
the block made.
"""
import pytest
import torch

from paper_2010_14298_gb300 import ffn, fqt


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")
class TestGatedBlock:
    def _data(self, T, D, seed=3):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        x = torch.randn(T, D, generator=g, device="cuda").bfloat16()
        return x, x.float() + 0.3 * torch.randn(T, D, generator=g, device="cuda")

    @pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "sigmoid"])
    @pytest.mark.parametrize("T,D,H", [(512, 256, 512), (300, 144, 400)])
    def test_a_step_matches_64_bits(self, T, D, H, act):
        x, target = self._data(T, D)
        block = ffn.GatedFfnBlock(T, D, H, act, max_norm=1e9)
        p = [t.double().detach().clone().requires_grad_() for t in block.parameters]
        xd = x.double().requires_grad_()
        mean = xd.mean(1, keepdim=True)
        var = ((xd - mean) ** 2).mean(1, keepdim=True)
        y = (xd - mean) * (var + 1e-5) ** -0.5 * p[3] + p[4]
        f = torch.nn.functional
        act64 = {"silu": f.silu, "gelu": f.gelu, "sigmoid": torch.sigmoid,
                 "gelu_tanh": lambda v: f.gelu(v, approximate="tanh")}[act]
        out = xd + (act64(y @ p[0].t()) * (y @ p[1].t())) @ p[2].t()
        loss = ((out - target.double()) ** 2).sum() / (2 * T)
        grads = torch.autograd.grad(loss, p + [xd])
        diff = block.forward(x) - target
        assert abs(float(diff.square().sum() / (2 * T)) / loss.item() - 1) < 0.05
        dx = block.backward(diff / T)
        assert block.check() == 0
        for g, ref in zip(list(block.grads) + [dx], grads):
            assert (g.double() - ref).norm() <= 0.15 * ref.norm()
        norm = sum(float(g.double().square().sum()) for g in block.grads) ** 0.5
        assert abs(float(block.norm) / norm - 1) < 1e-5

    def test_steps_change_every_parameter(self):
        x, target = self._data(300, 144)
        block = ffn.GatedFfnBlock(300, 144, 256)
        before = [p.clone() for p in block.parameters]
        for _ in range(2):
            block.step(x, target, 0.03)
        assert block.check() == 0
        for p, old in zip(block.parameters, before):
            assert p.isfinite().all() and not torch.equal(p, old)

    def test_the_same_bits_through_ctypes(self, monkeypatch):
        x, target = self._data(300, 128)
        first = ffn.GatedFfnBlock(300, 128, 256, "gelu")
        first.step(x, target, 0.01)
        monkeypatch.setattr(fqt, "_native", fqt._CtypesCalls(fqt.load()))
        second = ffn.GatedFfnBlock(300, 128, 256, "gelu")
        second.step(x, target, 0.01)
        assert second.check() == 0
        assert torch.equal(first.norm, second.norm)
        assert all(torch.equal(a, b) for a, b in zip(first.parameters, second.parameters))

    def test_command(self):
        ffn.main(["--tokens", "256", "--width", "128", "--hidden", "256", "--steps", "2", "--gated",
                  "gelu_tanh"])


def test_refusals():
    with pytest.raises(ValueError):
        ffn.GatedFfnBlock(16, 32, 32, "tanh")
    for argv in (["--gated", "tanh"], ["--gated", "silu", "--format", "int8"]):
        with pytest.raises(SystemExit):
            ffn.main(argv)
