"""The gated operators' activations far from zero, and over the whole range between.

g takes chosen values: a token holds two entries in blocks of their own (a large one and a
small one, or one alone) and the weights' ones pick them, so that g is their sum, exactly,
and u is 1.

Tolerances.  The exponential (ex2.approx: 2^-22 of itself) takes z log2 e, which is rounded
twice and is off by at most |z| 2^-23, the same of the result; z itself is off by four
roundings for gelu_tanh, |z| 2^-22 more, and g^2 / 2 by one for gelu.  The quotient
(rcp.approx) is off by 2^-23, gelu's polynomial by 3.2e-8 and 24 roundings of fp32.  Together
at most (24 + 10 z) 2^-24 of a value, z the largest argument of an exponential.  sigma is a
normal number of fp32 or 0, so an act(g) below 2^-126 (1 + |g|) may be 0.
"""
import math

import pytest
import torch

from paper_2010_14298_gb300 import fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = tuple(fqt.ACTIVATIONS)
TANH = 2 * math.sqrt(2 / math.pi)
FAR = [100.0, 1e3, 1e6, 1e20, 1e30, 1e35, 1e38, 3e38]
# few tokens (one CTA to a block, and four), tiles whose K blocks a cluster shares, narrow
# ones of a dense output, pairs of CTAs
SIZES = [(3, 60), (20, 300), (130, 300), (200, 4096), (2100, 1000)]


def _act(g, act):
    """act(g), act'(g) and the largest argument of an exponential, in 64 bits."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).double(), 0 * g
    if act == "gelu":
        cdf, phi = 0.5 * torch.erfc(-g / 2 ** 0.5), torch.exp(-g * g / 2) / (2 * math.pi) ** 0.5
        return g * cdf, cdf + g * phi, g * g / 2
    z = TANH * (g + 0.044715 * g ** 3) if act == "gelu_tanh" else g
    dz = TANH * (1 + 3 * 0.044715 * g * g) if act == "gelu_tanh" else torch.ones_like(g)
    s, r = torch.sigmoid(z), torch.sigmoid(-z)
    if act == "sigmoid":
        return s, s * r, z.abs()
    return g * s, s + g * s * r * dz, z.abs()


def _tokens(large, small, H, ws):
    """Operands for which g of a token is large + small (as codes hold them) and u is 1, and
    g in 64 bits."""
    T = large.numel()
    X = torch.zeros((T, 384), device="cuda")
    X[:, 0], X[:, 128], X[:, 256] = large, small, 1.0
    Wg, Wu = torch.zeros((2, H, 384), device="cuda")
    Wg[:, 0] = Wg[:, 128] = Wu[:, 256] = 1.0
    a, bg, bu = (fqt.quantize_fp8(x, b, ws=ws)[0] for x, b in ((X, 1), (Wg, 128), (Wu, 128)))
    v = a.dequantize().double()
    return a, bg, bu, (v[:, :1] + v[:, 128:129]).expand(T, H)


def _rows(values, T):
    v = torch.tensor(values, device="cuda")
    return v.repeat(-(-T // v.numel()))[:T]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,H", SIZES)
def test_forward_far_from_zero(T, H, act):
    """0 on the left (at -100 1e-30 and less), g or 1 on the right, to two units of the quotient and
    two roundings; the codes are those of the dense output."""
    ws = fqt.Workspace.of_size(256)
    v = _rows([x for f in FAR for x in (-f, f)], T)
    a, bg, bu, g = _tokens(v, torch.zeros_like(v), H, ws)
    want = _act(g, act)[0]
    for dtype in DTYPES.values():
        tol = 2.0 ** -22 + (2.0 ** -8 if dtype is torch.bfloat16 else 0)
        alone = fqt.fp8_gated_matmul(a, bg, bu, act, dtype=dtype, ws=ws)[0]
        out, q, gate, _ = fqt.fp8_gated_matmul(a, bg, bu, act, dtype=dtype, codes=True, keep=True, ws=ws)
        assert fqt.sync_status(ws) == 0
        for x in (alone, out):
            assert ((x.double() - want).abs() <= tol * want.abs() + 1e-30).all()
            assert (x[g <= -1e3] == 0).all()
        if dtype is torch.float32:
            ref = fqt.quantize_fp8(out)[0]
            assert torch.equal(q.codes[:, :H], ref.codes[:, :H])
        half = 2.0 ** -4  # a code's rounding
        assert ((gate.dequantize().double() - g).abs() <= half * g.abs()).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_far_from_zero(dtype, act):
    """The slope and the value: 0 on the left, 1 and g (sigmoid's 0 and 1) on the right."""
    dtype = DTYPES[dtype]
    v = _rows([x for f in FAR for x in (-f, f)], 64)
    g = v[:, None].expand(64, 200).contiguous()
    gate, up = fqt.quantize_fp8(g)[0], fqt.quantize_fp8(torch.ones_like(g))[0]
    dA = torch.ones_like(g).to(dtype)
    want, slope, _ = _act(gate.dequantize().double(), act)
    tol = 2.0 ** -22 + (2.0 ** -8 if dtype is torch.bfloat16 else 0)
    ws = fqt.Workspace.of_size(256)
    r = fqt.fp8_gated_backward(dA, gate, up, act, ws=ws, out=fqt.GatedGrads(
        dgate=torch.empty_like(dA), dup=torch.empty_like(dA)))
    for got, ref in ((r.dgate, slope), (r.dup, want)):
        assert ((got.double() - ref).abs() <= tol * ref.abs() + 1e-30).all()
        assert (got[v <= -1e3] == 0).all()
    codes = fqt.fp8_gated_backward(dA, gate, up, act, ws=ws)
    assert fqt.sync_status(ws) == 0
    # (a code's half step, relative or of the scale, which is at most a row's largest / 224)
    for q, ref in ((codes.qgate, slope), (codes.qup, want), (codes.product_t, want.t())):
        off = 2.0 ** -4 * ref.abs() + 2.0 ** -10 / 224 * ref.abs().amax(1, keepdim=True)
        assert ((q.dequantize().double() - ref).abs() <= 1.001 * off + 1e-30).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,H", [(64, 40), (1500, 40), (4096, 600)])
def test_forward_over_the_range(T, H, act):
    """g of up to 20 bits between -100 and 100 (gelu: 14, where its tail leaves fp32)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    top = 14.0 if act in ("gelu", "gelu_tanh") else 100.0
    large = (torch.rand(T, generator=gen, device="cuda") * 2 - 1) * top
    # (steps of 2^-14: with 3 bits after the large one's leading bit, at most 21 in all)
    small = torch.randint(-15, 16, (T,), generator=gen, device="cuda") * 2.0 ** -14
    ws = fqt.Workspace.of_size(256)
    a, bg, bu, g = _tokens(large, small, H, ws)
    want, _, z = _act(g, act)
    out = fqt.fp8_gated_matmul(a, bg, bu, act, ws=ws)[0]
    assert fqt.sync_status(ws) == 0
    tol = (24 + 10 * z) * 2.0 ** -24
    least = 2.0 ** -125 * (1 + g.abs())
    assert ((out.double() - want).abs() <= tol * want.abs() + least).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_checkpoint_that_is_no_number(dtype, act):
    """A NaN code among g's: dg, du and a are no numbers there, whichever of them is asked
    for, and it is recorded where they leave as codes."""
    T, H, i, j = 150, 300, 131, 290
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    g, u, dA = torch.randn((3, T, H), generator=gen, device="cuda")
    dA = dA.to(DTYPES[dtype])
    gate, up = fqt.quantize_fp8(g)[0], fqt.quantize_fp8(u)[0]
    gate.codes[i, j] = 0x7F
    ws = fqt.Workspace.of_size(256)
    r = fqt.fp8_gated_backward(dA, gate, up, act, ws=ws, out=fqt.GatedGrads(
        dgate=torch.empty_like(dA), dup=torch.empty_like(dA)))
    assert fqt.sync_status(ws) == 0  # as other dense outputs
    there = torch.zeros((T, H), dtype=torch.bool, device="cuda")
    there[i, j] = True
    assert torch.equal(r.dgate.isnan(), there) and torch.equal(r.dup.isnan(), there)
    for name in ("qgate", "qup", "qgate_t", "qup_t", "product_t"):
        n, k, at = (T, H, there) if name in ("qgate", "qup") else (H, T, there.t())
        q = fqt.Fp8Tensor.empty(n, k)
        fqt.fp8_gated_backward(dA, gate, up, act, out=fqt.GatedGrads(**{name: q}), ws=ws)
        assert fqt.sync_status(ws) == 4, name
        assert torch.equal(q.codes[:, :k] & 127 == 127, at), name
