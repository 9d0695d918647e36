"""A transformer's feed-forward block trained with this library's operators.

    y = x + W2 relu(W1 norm(x))

One training step is the layer norm, the two linear layers in a low-bit format,
their gradients, the norm's gradients, and the clipping of all gradients to a global
norm.  The linear layers run in 8-bit floating point with a scale per block of 128
("fp8"), or fully quantized ("int8": 8-bit activations and weights, 8-bit BHQ output
gradients, 8-bit stochastic gradients for the weights).  What these operators write is
allocated once; the ReLU, the residual sums and the loss between them are PyTorch's.

    python -m paper_2010_14298_gb300.ffn --tokens 8192 --width 1024 --hidden 4096
"""
from __future__ import annotations

import argparse

import torch

from . import fqt

FORMATS = ("fp8", "int8")


class _Fp8Linear:
    """H = X W^T and its gradients in 8-bit floating point."""

    def __init__(self, tokens, cols, rows, device):
        T, D, C = tokens, cols, rows
        Q = lambda r, c, b=1: fqt.Fp8Tensor.empty(r, c, b, device)  # noqa: E731
        bf16 = lambda *n: torch.empty(n, dtype=torch.bfloat16, device=device)  # noqa: E731
        self.qx, self.qxt = Q(T, D), Q(D, T)
        self.qw, self.qwt = Q(C, D, fqt.FP8_BLOCK), Q(D, C, fqt.FP8_BLOCK)
        self.qd, self.qdt = Q(T, C), Q(C, T)
        self.H, self.dX = bf16(T, C), bf16(T, D)
        self.dW = torch.empty((C, D), dtype=torch.float32, device=device)
        self.ws = fqt.Workspace.of_size(max(fqt.fp8_matmul_workspace_size(*s) for s in (
            (T, C, D), (T, D, C), (C, D, T))), device)

    def forward(self, X, W):
        fqt.quantize_fp8(X, q=self.qx, qt=self.qxt, ws=self.ws)
        fqt.quantize_fp8(W, fqt.FP8_BLOCK, q=self.qw, qt=self.qwt, ws=self.ws)
        return fqt.fp8_matmul(self.qx, self.qw, out=self.H, ws=self.ws)

    def backward(self, dH, seed):
        del seed  # nothing is rounded stochastically
        fqt.quantize_fp8(dH, q=self.qd, qt=self.qdt, ws=self.ws)
        fqt.fp8_matmul(self.qdt, self.qxt, out=self.dW, ws=self.ws)
        return fqt.fp8_matmul(self.qd, self.qwt, out=self.dX, ws=self.ws)

    def check(self):
        return fqt.sync_status(self.ws)


class _Int8Linear:
    """The same with integer codes: App. E's bifurcated gradients."""

    bits, block = 8, 16

    def __init__(self, tokens, cols, rows, device):
        T, D, C = tokens, cols, rows
        Q = fqt.QTensor.empty
        self.qx = Q(T, D, fqt.PTQ, 8, 0, True, True, device, u8=False)
        self.qw = Q(C, D, fqt.PTQ, 8, 0, True, True, device, u8=False)
        self.q2 = Q(T, C, fqt.BHQ, self.bits, self.block, True, False, device, u8=False)
        self.q1 = Q(T, C, fqt.PTQ, 8, 0, False, True, device, u8=False)
        f32 = lambda *n: torch.empty(n, dtype=torch.float32, device=device)  # noqa: E731
        self.H, self.dX, self.dW = f32(T, C), f32(T, D), f32(C, D)
        self.ws = fqt.Workspace(T, C, D, device)

    def forward(self, X, W):
        fqt.quantize_act(X, 8, ws=self.ws, out=self.qx, row_sum=True)
        fqt.quantize_weight(W, 8, ws=self.ws, out=self.qw, row_sum=True)
        return fqt.linear_forward(self.qx, self.qw, ws=self.ws, out=self.H)

    def backward(self, dH, seed):
        fqt.quantize_grad(dH, fqt.BHQ, self.bits, self.block, seed, ws=self.ws, q_b2=self.q2,
                          q_b1=self.q1)
        fqt.linear_backward(self.q2, self.q1, self.qx, self.qw, ws=self.ws, out_x=self.dX,
                            out_w=self.dW)
        return self.dX

    def check(self):
        return fqt.sync_status(self.ws)


class FfnBlock:
    """The block, its parameters in fp32 and the buffers of a step of `tokens` tokens."""

    def __init__(self, tokens: int, width: int, hidden: int, format: str = "fp8",
                 max_norm: float = 1.0, seed: int = 0, device="cuda"):
        if format not in FORMATS:
            raise ValueError(f"format is one of {FORMATS}, not {format!r}")
        if format == "int8" and (width % 16 or hidden % 16):
            raise ValueError("int8 layers have multiples of 16 columns")
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        randn = lambda *n: torch.randn(n, generator=g, device=device)  # noqa: E731
        self.W1 = randn(hidden, width) * (2.0 / width) ** 0.5
        self.W2 = randn(width, hidden) * (0.1 / hidden ** 0.5)
        self.gamma = torch.ones(width, device=device)
        self.beta = torch.zeros(width, device=device)
        linear = _Fp8Linear if format == "fp8" else _Int8Linear
        self.up = linear(tokens, width, hidden, device)
        self.down = linear(tokens, hidden, width, device)
        f32 = lambda *n: torch.empty(n, device=device)  # noqa: E731
        self.y = torch.empty((tokens, width), dtype=torch.bfloat16, device=device)
        self.mean, self.rstd = f32(tokens), f32(tokens)
        self.dx = torch.empty_like(self.y)
        self.dgamma, self.dbeta = f32(width), f32(width)
        self.grads = fqt.TensorList([self.up.dW, self.down.dW, self.dgamma, self.dbeta])
        self.norm, self.max_norm, self.steps = f32(1), max_norm, 0
        self.ws = fqt.Workspace.of_size(max(fqt.layer_norm_workspace_size(tokens, width),
                                            fqt.clip_grad_norm_workspace_size(self.grads)),
                                        device)

    @property
    def parameters(self):
        return [self.W1, self.W2, self.gamma, self.beta]

    def forward(self, x):
        """x (tokens x width, bf16) + the block's output, in fp32."""
        fqt.layer_norm_forward(x, self.gamma, self.beta, out=self.y, mean=self.mean,
                               rstd=self.rstd)
        self.x = x
        h = self.up.forward(self.y, self.W1)
        self.a = torch.relu(h).bfloat16()
        return x.float() + self.down.forward(self.a, self.W2).float()

    def backward(self, dout):
        """The gradients (in `grads`, clipped) and the input's, for the output's."""
        dout = dout.bfloat16()
        da = self.down.backward(dout, 2 * self.steps)
        dh = (da * (self.a > 0)).bfloat16()
        dy = self.up.backward(dh, 2 * self.steps + 1).bfloat16()
        fqt.layer_norm_backward(dy, self.x, self.mean, self.rstd, self.gamma, ws=self.ws,
                                out_x=self.dx, out_gamma=self.dgamma, out_beta=self.dbeta)
        fqt.clip_grad_norm(self.grads, self.max_norm, norm=self.norm, ws=self.ws)
        return dout + self.dx

    def step(self, x, target, lr: float):
        """One step on half the mean square error; returns the loss (on the GPU)."""
        diff = self.forward(x) - target
        self.backward(diff / x.shape[0])
        for p, g in zip(self.parameters, self.grads):
            p.add_(g, alpha=-lr)
        self.steps += 1
        return diff.square().sum() / (2 * x.shape[0])

    def check(self) -> int:
        """A condition that the kernels of the steps since the last call recorded, or 0
        (the up projection's before the down projection's, the norm's and the clipping's)."""
        states = [self.up.check(), self.down.check(), fqt.sync_status(self.ws)]
        return next((s for s in states if s), 0)


def main(argv=None):
    p = argparse.ArgumentParser(description="trains one feed-forward block on a fixed target")
    p.add_argument("--tokens", type=int, default=8192)
    p.add_argument("--width", type=int, default=1024)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--format", choices=FORMATS, default="fp8")
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--lr", type=float, default=0.03)
    p.add_argument("--max-norm", type=float, default=1.0)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(a.tokens, a.width, generator=g, device="cuda").bfloat16()
    mix = torch.randn(a.width, a.width, generator=g, device="cuda") / a.width ** 0.5
    target = x.float() + 0.3 * torch.relu(x.float() @ mix)
    block = FfnBlock(a.tokens, a.width, a.hidden, a.format, a.max_norm)
    times = []
    for i in range(a.steps):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        loss = block.step(x, target, a.lr)
        end.record()
        end.synchronize()
        times.append(start.elapsed_time(end))
        print(f"step {i}: loss {float(loss):.4f}, gradient norm {float(block.norm):.4f}")
    state = block.check()  # which clears it
    if state:
        raise SystemExit(f"a kernel recorded: {fqt.status_string(state)}")
    print(f"{a.format}: {sorted(times)[len(times) // 2]:.3f} ms a step")


if __name__ == "__main__":
    main()
