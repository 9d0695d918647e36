"""What is measured of the training-step operators around the quantized linear layers.

  op "norm"       layer norm of the rows of X (forward): Y and the rows' statistics
  op "norm_grad"  its backward pass: dX and the reductions of the scale's and the
                  shift's gradients over all rows
  op "linear"     a linear layer in 8-bit floating point (E4M3) with one scale for
                  each block of 128, the weight's codes kept between calls: X is
                  quantized, then H = X~ W~^T
  op "step"       a training step of such a layer: X, W and dY quantized along both
                  of their axes, H = X~ W~^T, grad_X = dY~ W~ and grad_W = dY~^T X~
  op "clip"       the global norm of a list of gradients, and the clipped gradients

``prepare`` draws the tensors, ``run`` is one pass, ``exact`` restates a pass in 64
bits. Where ``own`` is false a pass runs in elementary torch operations, in 32 bits.

The scale of a block is the least power of two 2^e (-127 <= e <= 127) for which no
entry exceeds 448, E4M3's largest value, after division by it; it is 1 for a block of
zeros. Entries are divided by it and rounded to the nearest E4M3 value, ties to even,
so the values that codes stand for are the same in any arithmetic. Blocks hold 128
consecutive entries of a row (activations and gradients) or 128 x 128 (weights), the
last ones what is left.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 128
EPS = 1e-5


# --------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------
def _norm(op, rows, cols, dtype, affine=True, gap=0, **name):
    """gap: X is the first cols columns of rows of cols + gap entries."""
    return dict(name, op=op, rows=rows, cols=cols, dtype=dtype, affine=affine, gap=gap)


def _linear(op, T, C, D, dtype, **name):
    return dict(name, op=op, T=T, C=C, D=D, dtype=dtype)


def _clip(kind, max_norm, dtype, count=0, total=0, shapes=0, **name):
    return dict(name, op="clip", kind=kind, max_norm=max_norm, dtype=dtype, count=count,
                total=total, shapes=shapes)


def listed():
    return [
        # one token at the FFN's width, as in generation: the cost of a call
        _norm("norm", 1, 1024, "bf16", name="norm_1x1024_bf16"),
        # the norm before the FFN at 8192 tokens
        _norm("norm", 8192, 1024, "bf16", name="norm_8192x1024_bf16"),
        # rows of odd length inside a wider projection: nothing is aligned
        _norm("norm", 1523, 1201, "f32", gap=402, name="norm_1523x1201_f32_strided"),
        # gradients of the FFN's norm at 8192 tokens
        _norm("norm_grad", 8192, 1024, "bf16", name="norm_grad_8192x1024_bf16"),
        # a narrow norm of few, oddly long rows
        _norm("norm_grad", 1523, 335, "f32", name="norm_grad_1523x335_f32"),
        # a wide norm over a large batch: memory traffic alone
        _norm("norm_grad", 32768, 4096, "bf16", name="norm_grad_32768x4096_bf16"),
        # one token through the FFN's up projection, weights kept as codes
        _linear("linear", 1, 4096, 1024, "bf16", name="linear_1x4096x1024_bf16"),
        # the FFN's down projection of 8192 tokens in evaluation
        _linear("linear", 8192, 1024, 4096, "bf16", name="linear_8192x1024x4096_bf16"),
        # a layer of no convenient size: ragged blocks in every dimension
        _linear("step", 1523, 336, 1201, "f32", name="step_1523x336x1201_f32"),
        # the FFN's up projection at 8192 tokens, forward and backward
        _linear("step", 8192, 4096, 1024, "bf16", name="step_8192x4096x1024_bf16"),
        # the gradients of one FFN block in bf16: four tensors
        _clip("ffn", 1.0, "bf16", name="clip_ffn_bf16"),
        # the gradients of a ResNet-50: 161 tensors of 64 to 2.4 million entries
        _clip("resnet50", 1.0, "f32", name="clip_resnet50_f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges, no larger than the largest of them."""
    op = rng.choice(["norm", "norm_grad", "linear", "step", "step", "clip"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("norm", "norm_grad"):
        while True:
            rows, cols = _log(rng, 1, 32768), _log(rng, 16, 8192)
            if rng.random() < 0.5:  # the widths that models mostly have
                cols = max(16, cols // 64 * 64)
            if rows * cols <= 1 << 26:
                break
        return _norm(op, rows, cols, dtype, affine=rng.random() < 0.8,
                     gap=rng.choice([0, 0, 7, 64]))
    if op == "clip":
        return _clip("drawn", rng.choice([0.01, 1.0, 1e6]), dtype, count=_log(rng, 1, 300),
                     total=_log(rng, 2000, 30_000_000), shapes=rng.randrange(1 << 30))
    while True:
        T, C, D = _log(rng, 1, 8192), _log(rng, 16, 4096), _log(rng, 16, 4096)
        if rng.random() < 0.5:
            C, D = max(16, C // 16 * 16), max(16, D // 16 * 16)
        if T * C * D <= 1 << 35:
            return _linear(op, T, C, D, dtype)


def _resnet50():
    """The parameter counts of a ResNet-50: 53 convolutions with a scale and a shift
    each, and the classifier."""
    counts = [64 * 3 * 49, 64, 64]
    cin = 64
    for width, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for b in range(blocks):
            for n, c in ((cin * width, width), (9 * width * width, width),
                         (4 * width * width, 4 * width)):
                counts += [n, c, c]
            if b == 0:
                counts += [cin * 4 * width, 4 * width, 4 * width]
            cin = 4 * width
    return counts + [1000 * 2048, 1000]


def _counts(case):
    if case["kind"] == "ffn":
        return [4096 * 1024, 1024 * 4096, 1024, 1024]
    if case["kind"] == "resnet50":
        return _resnet50()
    # sizes as models have them: a few large tensors, many small ones
    rng = random.Random(case["shapes"])
    weights = [math.exp(2.5 * rng.gauss(0, 1)) for _ in range(case["count"])]
    return [max(1, int(case["total"] * w / sum(weights))) for w in weights]


def work(case):
    """Each tensor that a user hands in read once, each one handed back written
    once. Codes that a pass makes stay inside; the kept weight's are read."""
    e = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op in ("norm", "norm_grad"):
        n, r, c = case["rows"] * case["cols"], case["rows"], case["cols"]
        vec = 2 if case["affine"] else 0
        if op == "norm":
            return {"bytes": 2 * n * e + 8 * r + 4 * vec * c, "flops": 8 * n}
        return {"bytes": 3 * n * e + 8 * r + (12 * c if vec else 0), "flops": 14 * n}
    if op == "clip":
        n = sum(_counts(case))
        return {"bytes": 2 * n * e + 4, "flops": 3 * n}
    T, C, D = case["T"], case["C"], case["D"]
    if op == "linear":
        kept = C * D + 4 * C * math.ceil(D / BLOCK) / BLOCK
        return {"bytes": T * D * e + kept + T * C * e, "flops": 2 * T * C * D}
    return {"bytes": (2 * T * D + 2 * T * C + C * D) * e + 4 * C * D, "flops": 6 * T * C * D}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
def _inputs(case, seed):
    """The tensors of a pass, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    t = TYPES[case["dtype"]]
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    op = case["op"]
    if op in ("norm", "norm_grad"):
        # activations: every channel with a mean and a size of its own, a few far
        # larger than the rest; gradients with lognormal rows
        rows, cols = case["rows"], case["cols"]
        X = randn(rows, cols + case["gap"])
        size = torch.exp(0.5 * randn(cols + case["gap"]))
        size[:: 97] *= 8.0
        X.mul_(size).add_(0.5 * randn(cols + case["gap"]))
        d = dict(X=X.to(t)[:, :cols])
        d["gamma"] = 1 + 0.2 * randn(cols) if case["affine"] else None
        d["beta"] = 0.1 * randn(cols) if case["affine"] else None
        if op == "norm_grad":
            d["dY"] = (randn(rows, cols) * torch.exp(randn(rows, 1))).to(t)
            x = d["X"].float()
            mean = x.mean(1, keepdim=True)
            rstd = torch.rsqrt((x - mean).square_().mean(1) + EPS)
            d.update(mean=mean.view(-1), rstd=rstd)
        return d
    if op == "clip":
        # tensors of different magnitudes; their norm is a few units
        counts = _counts(case)
        size = 4.0 / math.sqrt(sum(counts))
        return dict(grads=[(randn(n) * (size * math.exp(0.5 * math.sin(i)))).to(t)
                           for i, n in enumerate(counts)])
    # tokens with outlier channels, a small weight, gradients with lognormal rows
    T, C, D = case["T"], case["C"], case["D"]
    size = torch.exp(0.3 * randn(D))
    size[:: 211] *= 20.0
    d = dict(X=(randn(T, D) * size).to(t), W=(0.02 * randn(C, D)).to(t))
    if op == "step":
        d["dY"] = (1e-3 * randn(T, C) * torch.exp(1.5 * randn(T, 1))).to(t)
    return d


def prepare(case, seed):
    """The tensors of a pass, the outputs' buffers, and what a program keeps from
    call to call: the weight's codes of a layer in evaluation, the lists of
    gradients, and (with the framework) its code tensors and workspace."""
    d = _inputs(case, seed)
    op, t = case["op"], TYPES[case["dtype"]]
    s = dict(d, case=dict(case))
    if op == "clip":
        # the clipped gradients go into one buffer, each tensor on 16 bytes
        at, total = [], 0
        for g in d["grads"]:
            at.append(total)
            total += -(-g.numel() // 8) * 8
        s["flat"] = torch.zeros(total, dtype=t, device="cuda")
        s["out"] = [s["flat"][a:a + g.numel()] for a, g in zip(at, d["grads"])]
    elif op == "linear" and not own:
        s["W"] = _quantized(d["W"], weight=True)
    if own:
        from paper_2010_14298_gb300 import fqt
        empty = lambda *n, dt=t: torch.empty(n, dtype=dt, device="cuda")  # noqa: E731
        s["fqt"] = fqt
        if op in ("norm", "norm_grad"):
            rows, cols = case["rows"], case["cols"]
            f32 = torch.float32
            if op == "norm":
                s.update(y=empty(rows, cols), mean_out=empty(rows, dt=f32),
                         rstd_out=empty(rows, dt=f32))
            else:
                s.update(dx=empty(rows, cols), ws=fqt.Workspace.of_size(
                    fqt.layer_norm_workspace_size(rows, cols)))
                s.update(dgamma=empty(cols, dt=f32) if case["affine"] else None,
                         dbeta=empty(cols, dt=f32) if case["affine"] else None)
        elif op == "clip":
            s.update(grads=fqt.TensorList(d["grads"]), out=fqt.TensorList(s["out"]),
                     norm=empty(1, dt=torch.float32))
            s["ws"] = fqt.Workspace.of_size(fqt.clip_grad_norm_workspace_size(s["grads"]))
        else:
            T, C, D = case["T"], case["C"], case["D"]
            Q = fqt.Fp8Tensor.empty
            s.update(qx=Q(T, D), qw=Q(C, D, BLOCK), H=empty(T, C))
            s["ws"] = fqt.Workspace.of_size(max(fqt.fp8_matmul_workspace_size(T, C, D),
                                                fqt.fp8_matmul_workspace_size(T, D, C),
                                                fqt.fp8_matmul_workspace_size(C, D, T)))
            if op == "linear":
                fqt.quantize_fp8(d["W"], block_rows=BLOCK, q=s["qw"], ws=s["ws"])
                del s["W"]
            else:
                s.update(qxt=Q(D, T), qwt=Q(D, C, BLOCK), qd=Q(T, C), qdt=Q(C, T),
                         gx=empty(T, D), gw=empty(C, D, dt=torch.float32))
    return s


# --------------------------------------------------------------------------
# One pass in elementary operations
# --------------------------------------------------------------------------
def _pow2(e):
    """2^e for -127 <= e <= 127, by its bits (powers are rounded)."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).int().view(torch.float32)


def _blocked(x, weight):
    """x, padded to whole blocks, as (row blocks, block rows, column blocks, 128)."""
    rows, cols = x.shape
    br = BLOCK if weight else 1
    R, K = -(-rows // br), -(-cols // BLOCK)
    padded = torch.zeros((R * br, K * BLOCK), dtype=x.dtype, device=x.device)
    padded[:rows, :cols] = x
    return padded.view(R, br, K, BLOCK)


def _quantized(x, weight=False):
    """The codes and the scales of x along its rows, in blocks."""
    b = _blocked(x.float(), weight)
    m, e = torch.frexp(b.abs().amax((1, 3), keepdim=True))
    e = torch.clamp(torch.where(m > 0.875, e - 8, e - 9), -127, 127)
    e = torch.where(m > 0, e, torch.zeros_like(e))
    return (b * _pow2(-e)).to(torch.float8_e4m3fn), e, tuple(x.shape)


def _values(q):
    codes, e, (rows, cols) = q
    b = codes.float() * _pow2(e)
    return b.reshape(b.shape[0] * b.shape[1], -1)[:rows, :cols]


def _plain(s):
    c, t = s["case"], TYPES[s["case"]["dtype"]]
    op = c["op"]
    if op == "norm":
        x = s["X"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt(d.square().mean(1, keepdim=True) + EPS)
        y = d * rstd
        if c["affine"]:
            y = y * s["gamma"] + s["beta"]
        return {"y": y.to(t), "mean": mean.view(-1), "rstd": rstd.view(-1)}
    if op == "norm_grad":
        dy, rstd = s["dY"].float(), s["rstd"][:, None]
        xhat = (s["X"].float() - s["mean"][:, None]) * rstd
        g = dy * s["gamma"] if c["affine"] else dy
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        out = {"dx": dx.to(t)}
        if c["affine"]:
            out.update(dgamma=(dy * xhat).sum(0), dbeta=dy.sum(0))
        return out
    if op == "clip":
        squares = [g.float().square().sum() for g in s["grads"]]
        norm = torch.stack(squares).sum().sqrt()
        scale = torch.where(norm > c["max_norm"], c["max_norm"] / norm, torch.ones_like(norm))
        [o.copy_(g.float() * scale) for o, g in zip(s["out"], s["grads"])]
        return {"norm": norm.view(1), "grads": s["flat"]}
    x = _values(_quantized(s["X"]))
    if op == "linear":
        return {"H": (x @ _values(s["W"]).T).to(t)}
    w, dy = _values(_quantized(s["W"], weight=True)), _values(_quantized(s["dY"]))
    xt, dyt = _values(_quantized(s["X"].T)), _values(_quantized(s["dY"].T))
    return {"H": (x @ w.T).to(t), "grad_X": (dy @ w).to(t), "grad_W": dyt @ xt.T}


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(s):
    if not own:
        return _plain(s)
    c, fqt = s["case"], s["fqt"]
    op = c["op"]
    if op == "norm":
        y, mean, rstd = fqt.layer_norm_forward(s["X"], s["gamma"], s["beta"], EPS, out=s["y"],
                                               mean=s["mean_out"], rstd=s["rstd_out"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        dx, dgamma, dbeta = fqt.layer_norm_backward(
            s["dY"], s["X"], s["mean"], s["rstd"], s["gamma"], ws=s["ws"], out_x=s["dx"],
            out_gamma=s["dgamma"], out_beta=s["dbeta"], grad_w=c["affine"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op == "clip":
        norm = fqt.clip_grad_norm(s["grads"], c["max_norm"], out=s["out"], norm=s["norm"],
                                  ws=s["ws"])
        return {"norm": norm, "grads": s["flat"]}
    if op == "linear":
        fqt.quantize_fp8(s["X"], q=s["qx"], ws=s["ws"])
        return {"H": fqt.fp8_matmul(s["qx"], s["qw"], out=s["H"], ws=s["ws"])}
    ws = s["ws"]
    fqt.quantize_fp8(s["X"], q=s["qx"], qt=s["qxt"], ws=ws)
    fqt.quantize_fp8(s["W"], block_rows=BLOCK, q=s["qw"], qt=s["qwt"], ws=ws)
    H = fqt.fp8_matmul(s["qx"], s["qw"], out=s["H"], ws=ws)
    fqt.quantize_fp8(s["dY"], q=s["qd"], qt=s["qdt"], ws=ws)
    gx = fqt.fp8_matmul(s["qd"], s["qwt"], out=s["gx"], ws=ws)
    gw = fqt.fp8_matmul(s["qdt"], s["qxt"], out=s["gw"], ws=ws)
    return {"H": H, "grad_X": gx, "grad_W": gw}


# --------------------------------------------------------------------------
# The same pass in 64 bits
# --------------------------------------------------------------------------
def _two_to(e):
    """2^e in 64 bits, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(v):
    """The nearest E4M3 values of v (|v| <= 448), ties to even: 3 bits below the
    leading one, steps of 2^-9 under 2^-6."""
    _, e = torch.frexp(v)
    step = _two_to(torch.clamp(e - 4, min=-9))
    return torch.round(v / step) * step


def _coded(x, weight=False):
    """What the codes of x stand for, its blocks along the rows."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    for k in range(0, cols, BLOCK):
        part = x[:, k:k + BLOCK]
        amax = part.abs().amax(1)
        if weight:
            whole = torch.zeros(-(-rows // BLOCK) * BLOCK, dtype=x.dtype, device=x.device)
            whole[:rows] = amax
            amax = whole.view(-1, BLOCK).amax(1).repeat_interleave(BLOCK)[:rows]
        e = torch.ceil(torch.log2(amax.clamp(min=1e-45) / 448))
        # log2 is rounded: the exponent is set right by comparison
        e = torch.where(_two_to(e) * 448 < amax, e + 1, e)
        e = torch.where(_two_to(e - 1) * 448 >= amax, e - 1, e)
        e = torch.where(amax > 0, e.clamp(-127, 127), torch.zeros_like(e))
        scale = _two_to(e)[:, None]
        out[:, k:k + BLOCK] = _e4m3(part / scale) * scale
    return out


def exact(case, seed):
    d = _inputs(case, seed)
    op = case["op"]
    wide = lambda k: d[k].double() if d.get(k) is not None else None  # noqa: E731
    if op in ("norm", "norm_grad"):
        x, gamma = wide("X"), wide("gamma")
        if op == "norm":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = (var + EPS) ** -0.5
            y = (x - mean[:, None]) * rstd[:, None]
            y = y if gamma is None else torch.addcmul(wide("beta"), y, gamma)
            return {"y": y, "mean": mean, "rstd": rstd}
        dy, rstd = wide("dY"), wide("rstd")[:, None]
        xhat = (x - wide("mean")[:, None]) * rstd
        g = dy if gamma is None else dy * gamma
        n = x.shape[1]
        dot = torch.einsum("ij,ij->i", g, xhat)[:, None]
        dx = rstd / n * (n * g - g.sum(1, keepdim=True) - xhat * dot)
        if gamma is None:
            return {"dx": dx}
        return {"dx": dx, "dgamma": torch.einsum("ij,ij->j", dy, xhat), "dbeta": dy.sum(0)}
    if op == "clip":
        grads = [g.double() for g in d["grads"]]
        norm = math.sqrt(math.fsum(float(torch.dot(g, g)) for g in grads))
        scale = min(1.0, case["max_norm"] / norm) if norm > 0 else 1.0
        parts = []
        for g in grads:
            parts.append(torch.zeros(-(-g.numel() // 8) * 8, dtype=torch.float64, device="cuda"))
            parts[-1][:g.numel()] = g * scale
        return {"norm": torch.full((1,), norm, dtype=torch.float64), "grads": torch.cat(parts)}
    x, w = wide("X"), wide("W")
    H = _coded(x) @ _coded(w, weight=True).T
    if op == "linear":
        return {"H": H}
    dy = wide("dY")
    return {"H": H, "grad_X": _coded(dy) @ _coded(w, weight=True),
            "grad_W": _coded(dy.T.contiguous()) @ _coded(x.T.contiguous()).T}
