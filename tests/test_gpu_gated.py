"""The gated feed-forward block's operators against plain implementations in 64 bits.

Tolerances.  A sum over K entries is off by at most e = (K / 32 + 20) 2^-23 S, S the sum
of its terms' magnitudes: a step of 32 terms drops under 2^-23 of the accumulator.  The
exponential that the activations take is off by (2 + 1.16 |z|) 2^-23 of itself (CUDA's bound
for __expf), the quotient by two units, z by a few roundings of its own, the normal
distribution function by five units: together at most (24 + 10 z) 2^-24 of the terms'
magnitudes, z the largest argument of an exponential.  Slopes are at most 1.13, so
a = act(g) u is off by |u| (1.13 e_g + E) + |act| e_u + 1.13 e_g e_u and a rounding to fp32.
A rounding to bf16 adds 2^-8 of the value.  Codes are exact: those of the same call's fp32
outputs, or of sums of small integers, which fp32 holds exactly.
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


def _randn(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


def _f8(x, block_rows=1):
    return fqt.quantize_fp8(x, block_rows)[0]


def _operands(T, H, K, size=1.0):
    """Tokens and both weights; g and u of size 1."""
    X = _randn(T, K, seed=1) * torch.exp(_randn(T, 1, seed=2)) * size
    return _f8(X), *(_f8(_randn(H, K, seed=s) / K ** 0.5, 128) for s in (3, 4))


def _sums(a, b):
    A, B = a.dequantize().double(), b.dequantize().double()
    return A @ B.t(), (A.abs() @ B.abs().t()) * ((A.shape[1] / 32 + 20) * 2.0 ** -23)


def _act(g, act):
    """act(g), act'(g), and the magnitudes of their terms times (24 + 10 z) 2^-24."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).double(), 0 * g, 0 * g
    if act == "gelu":
        cdf, phi = 0.5 * torch.erfc(-g / 2 ** 0.5), torch.exp(-g * g / 2) / (2 * math.pi) ** 0.5
        e = (24 + 5 * g * g) * 2.0 ** -24
        return g * cdf, cdf + g * phi, 24 * 2.0 ** -24 * (g * cdf).abs(), e * (cdf + (g * phi).abs())
    z = TANH * (g + 0.044715 * g ** 3) if act == "gelu_tanh" else g
    dz = TANH * (1 + 3 * 0.044715 * g * g) if act == "gelu_tanh" else torch.ones_like(g)
    s = torch.sigmoid(z)
    # (a sigma below fp32's normal numbers may be 0)
    e, least = (24 + 10 * z.abs()) * 2.0 ** -24, 2.0 ** -120
    if act == "sigmoid":
        return s, s * (1 - s), e * s + least, e * s * (1 - s) + least
    r = torch.sigmoid(-z)
    return (g * s, s + g * s * r * dz, (e * s + least) * g.abs(),
            e * (s + (g * s * r * dz).abs()) + least * (1 + g.abs()))


def _expected(a, bg, bu, act):
    """g, u, act(g) u and the largest error of the latter in fp32."""
    (g, eg), (u, eu) = _sums(a, bg), _sums(a, bu)
    v, _, E, _ = _act(g, act)
    out = v * u
    return g, u, out, (u.abs() * (1.13 * eg + E) + v.abs() * eu + 1.13 * eg * eu
                       + (E + 2.0 ** -24 * v.abs()) * (u.abs() + eu))


def _same(q, want):
    """The same codes and scales.  (Quantizing what codes stand for again is no such test: a
    block whose maximum was rounded down to 448 2^e takes the next smaller scale.)"""
    assert q.shape == want.shape
    assert torch.equal(q.codes[:, :q.cols], want.codes[:, :q.cols])
    nb = -(-q.cols // 128)
    scales = lambda t: t.scales.permute(0, 2, 1).reshape(-1, t.scales.shape[1])[:nb, :q.rows]  # noqa: E731
    assert torch.equal(scales(q), scales(want))


def _codes_equal(q, x):
    """q holds the codes of x (exactly)."""
    _same(q, _f8(x))


# few tokens; single CTAs; both with K blocks that a cluster shares; pairs of CTAs
SIZES = [(3, 300, 4000), (50, 40, 3000), (64, 1500, 1100), (130, 130, 4100), (70, 257, 2000),
         (400, 300, 1300), (1, 1, 1), (1, 4096, 1024), (2, 130, 27), (5, 5000, 300), (31, 335, 129), (33, 40, 700),
         (64, 128, 1201), (64, 700, 128), (65, 128, 64), (100, 17, 513), (129, 257, 1025),
         (300, 335, 1201), (700, 1000, 40), (2000, 1001, 200), (4111, 600, 96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,K", SIZES)
def test_forward_matches_64_bits(T, H, K, dtype):
    a, bg, bu = _operands(T, H, K)
    ws = fqt.Workspace.of_size(fqt.fp8_gated_matmul_workspace_size(T, H, K))
    for act in ACTS:
        _, _, want, bound = _expected(a, bg, bu, act)
        if dtype == "bf16":
            bound = bound + 2.0 ** -8 * (want.abs() + bound)
        out, q, gate, up = fqt.fp8_gated_matmul(a, bg, bu, act, dtype=DTYPES[dtype], ws=ws)
        assert fqt.sync_status(ws) == 0
        assert out.dtype == DTYPES[dtype] and out.shape == (T, H) and q is gate is up is None
        assert ((out.double() - want).abs() <= bound).all(), act


@pytest.mark.parametrize("T,H,K", [(1, 200, 2000), (40, 300, 1100), (90, 130, 3000),
                                   (300, 400, 2600), (2100, 1000, 1200)])
def test_long_sums(T, H, K):
    """More K blocks than an accumulator of an fp32 output takes."""
    a, bg, bu = _operands(T, H, K)
    _, _, want, bound = _expected(a, bg, bu, "silu")
    out = fqt.fp8_gated_matmul(a, bg, bu, "silu")[0]
    assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("T,H", [(70, 130), (2100, 1000), (20, 130)])
def test_long_sums_in_bf16(T, H):
    """More K blocks than an accumulator of a bf16 output takes."""
    a, bg, bu = _operands(T, H, 8400)
    _, _, want, bound = _expected(a, bg, bu, "silu")
    out = fqt.fp8_gated_matmul(a, bg, bu, "silu", dtype=torch.bfloat16)[0]
    assert ((out.double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all()


@pytest.mark.parametrize("T,H,K", SIZES + [(3, 9000, 64), (40, 9000, 200)])
def test_codes_are_those_of_the_sums(T, H, K):
    """Small integers: g and u are exact in fp32, and so is relu(g) u."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    ints = lambda r, c, b: _f8(torch.randint(-4, 5, (r, c), generator=g, device="cuda").float(), b)  # noqa: E731
    a, bg, bu = ints(T, K, 1), ints(H, K, 128), ints(H, K, 128)
    A, G, U = (t.dequantize() for t in (a, bg, bu))
    gate64, up64 = A.double() @ G.double().t(), A.double() @ U.double().t()
    ws = fqt.Workspace.of_size(256)
    out, q, gate, up = fqt.fp8_gated_matmul(a, bg, bu, "relu", codes=True, keep=True, ws=ws)
    assert fqt.sync_status(ws) == 0
    assert torch.equal(out.double(), (gate64.clamp(min=0) * up64).float().double())
    _codes_equal(q, out)
    _codes_equal(gate, gate64.float())
    _codes_equal(up, up64.float())
    # each alone, and without the dense output
    for name, ref in (("q", q), ("gate", gate), ("up", up)):
        t = fqt.Fp8Tensor.empty(T, H)
        none = fqt.fp8_gated_matmul(a, bg, bu, "relu", dense=False, **{name: t})
        assert none[0] is None
        _same(t, ref)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,H,K", [(1, 4096, 128), (50, 200, 300), (200, 335, 1201), (2000, 1000, 130)])
def test_codes_are_those_of_the_dense_output(T, H, K, act):
    a, bg, bu = _operands(T, H, K)
    out, q, gate, up = fqt.fp8_gated_matmul(a, bg, bu, act, codes=True, keep=True)
    _codes_equal(q, out)
    # g and u lie where the codes say: half a step, 2^-4 of the value or 2^-10 of the scale
    g, u, _, _ = _expected(a, bg, bu, act)
    for t, x, e in ((gate, g, _sums(a, bg)[1]), (up, u, _sums(a, bu)[1])):
        s = _f8(x.abs().float()).scales  # (only its shape)
        assert s.shape == t.scales.shape
        e8 = t.scales[:, :T].permute(1, 0, 2).reshape(T, -1).int() - 127
        scale = torch.exp2(e8.double()).repeat_interleave(128, 1)[:, :H]
        half = torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * scale)
        assert ((t.dequantize().double() - x).abs() <= half + 1.07 * e).all()


@pytest.mark.parametrize("T,H,K", [(7, 200, 100), (7, 200, 3000), (64, 5000, 64), (130, 300, 200),
                                   (130, 300, 4200), (2100, 1000, 300)])
def test_any_choice_of_outputs(T, H, K):
    """Each of the 15 choices among a, its codes, g's and u's gives what all of them together
    give.  Its tiles may be others and sum in another order, so a sum's last bits may differ, by
    2^-20 of it or so, and a code where that much decides: one entry in 2^15, and by one step.
    Two and one in 1000 are allowed."""
    a, bg, bu = _operands(T, H, K)
    out, *ref = fqt.fp8_gated_matmul(a, bg, bu, "gelu_tanh", codes=True, keep=True)
    _, _, want, bound = _expected(a, bg, bu, "gelu_tanh")
    for choice in range(1, 16):
        qs = [fqt.Fp8Tensor.empty(T, H) if choice >> i & 1 else None for i in range(3)]
        wide = torch.full((T + 1, H + 5), 7.0, device="cuda") if choice & 8 else None
        dense = None if wide is None else wide[:T, :H]
        got = fqt.fp8_gated_matmul(a, bg, bu, "gelu_tanh", out=dense, q=qs[0], gate=qs[1], up=qs[2],
                                   dense=False)
        assert [x is None for x in got] == [not choice & b for b in (8, 1, 2, 4)]
        if wide is not None:
            assert ((dense.double() - want).abs() <= bound).all()
            assert (wide[T:] == 7).all() and (wide[:, H:] == 7).all()
        for t, r in zip(qs, ref):
            if t is not None:
                x, y = t.dequantize(), r.dequantize()
                assert (x != y).sum() <= 2 + T * H // 1000
                # (a step is 2^-9 of the scale near zero, and the scale at most a block's
                # largest entry / 224)
                step = 2.0 ** -3 * torch.maximum(x.abs(), y.abs()) + 2.0 ** -9 / 224 * y.abs().amax(1, keepdim=True)
                assert ((x - y).abs() <= step).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,K", [(70, 45, 300), (100, 59, 27), (300, 335, 330), (900, 1001, 64),
                                   (70, 45, 2000), (2100, 1005, 130), (20, 45, 2000)])
def test_dense_outputs_alone_in_wider_rows(T, H, K, dtype):
    a, bg, bu = _operands(T, H, K)
    _, _, want, bound = _expected(a, bg, bu, "silu")
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    for gap in (1, 3, 8):
        wide = torch.full((T + 1, H + gap), 7.0, dtype=DTYPES[dtype], device="cuda")
        fqt.fp8_gated_matmul(a, bg, bu, "silu", out=wide[:T, :H])
        assert ((wide[:T, :H].double() - want).abs() <= bound).all(), gap
        assert (wide[T:] == 7).all() and (wide[:, H:] == 7).all(), gap


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H,K", [(3, 131, 27), (60, 45, 129), (130, 59, 27), (300, 1201, 330),
                                   (2100, 1005, 130)])
def test_nothing_past_the_rows_is_read_or_written(T, H, K, dtype):
    a, bg, bu = _operands(T, H, K)
    for t in (a, bg, bu):
        t.codes[:, K:] = 0x7F  # not a number
        t.scales[:, t.rows:] = 255
        t.scales[K // 512:, :, -(-K // 128) % 4 or 4:] = 255
    _, _, want, bound = _expected(a, bg, bu, "silu")
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    pitch = -(-H // 16) * 16 + 32
    for gap in (1, 2, 3, 8):
        wide = torch.full((T + 1, H + gap), 7.0, dtype=DTYPES[dtype], device="cuda")
        bytes_ = [torch.full((T + 2, pitch), 0x55, dtype=torch.uint8, device="cuda")
                  for _ in range(3)]
        qs = [fqt.Fp8Tensor(b[:T], torch.empty(fqt.Fp8Tensor.scale_shape(T, H),
                                               dtype=torch.uint8, device="cuda"), T, H)
              for b in bytes_]
        ws = fqt.Workspace.of_size(256)
        fqt.fp8_gated_matmul(a, bg, bu, "silu", out=wide[:T, :H], q=qs[0], gate=qs[1], up=qs[2],
                             ws=ws)
        assert fqt.sync_status(ws) == 0
        assert ((wide[:T, :H].double() - want).abs() <= bound).all(), gap
        assert (wide[T:] == 7).all() and (wide[:, H:] == 7).all(), gap
        for b in bytes_:
            assert (b[T:] == 0x55).all() and (b[:, -(-H // 16) * 16:] == 0x55).all()
        if dtype == "f32":
            _codes_equal(qs[0], wide[:T, :H])


def test_entries_that_are_not_finite():
    """A token that is no number, and sums past fp32's range: recorded where codes are
    asked for; no other token changes."""
    for T, H in ((3, 300), (100, 300), (2000, 1000)):
        a, bg, bu = _operands(T, H, 256)
        ref = fqt.fp8_gated_matmul(a, bg, bu, "silu", codes=True, keep=True)
        a.codes[1, 5] = 0x7F
        ws = fqt.Workspace.of_size(256)
        out = fqt.fp8_gated_matmul(a, bg, bu, "silu", ws=ws)[0]
        assert fqt.sync_status(ws) == 0  # as a product's dense output
        assert out[1].isnan().all()
        got = fqt.fp8_gated_matmul(a, bg, bu, "silu", codes=True, keep=True, ws=ws)
        assert fqt.sync_status(ws) == 4
        rest = [i for i in range(T) if i != 1]
        assert torch.equal(got[0][rest], ref[0][rest])
        for t, r in zip(got[1:], ref[1:]):
            assert (t.codes[1, :H] & 127 == 127).all()
            assert torch.equal(t.dequantize()[rest], r.dequantize()[rest])
        # one column of u past the range: infinite there, its block's others keep their scale
        a, bg, bu = _operands(T, H, 256)
        a.scales.fill_(127), bg.scales.fill_(127), bu.scales.fill_(127)
        a.codes[0].fill_(0x38), bu.codes[7].fill_(0x7E)  # 1 and 448
        bu.scales[:, 7] = 254
        want = fqt.fp8_gated_matmul(a, bg, bu, "relu")[0]
        assert fqt.fp8_matmul(a, bu)[0, 7].isinf()
        out, q, gate, up = fqt.fp8_gated_matmul(a, bg, bu, "relu", codes=True, keep=True, ws=ws)
        assert fqt.sync_status(ws) == 4
        assert torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0))
        assert up.codes[0, 7] & 127 == 127
        fine = out[0].isfinite()
        masked = torch.where(fine, out[0], torch.zeros_like(out[0]))[None]
        assert torch.equal(q.dequantize()[0][fine], _f8(masked).dequantize()[0][fine])
        assert (q.codes[0, :H][~fine] & 127 == 127).all()


# --- backward ---------------------------------------------------------------
def _kept(T, H, size=1.5):
    g, u = _randn(T, H, seed=7) * size, _randn(T, H, seed=8)
    dA = 1e-3 * _randn(T, H, seed=9) * torch.exp(1.5 * _randn(T, 1, seed=10))
    return _f8(g), _f8(u), dA


def _backward64(dA, gate, up, act):
    d, g, u = dA.double(), gate.dequantize().double(), up.dequantize().double()
    v, slope, E, ES = _act(g, act)
    dg, du = d * u * slope, d * v
    r = 2.0 ** -22
    return (dg, (d * u).abs() * ES + r * dg.abs() + 2.0 ** -120,
            du, d.abs() * E + r * du.abs() + 2.0 ** -120)


BACK = [(1, 1), (1, 4096), (3, 130), (64, 128), (127, 129), (128, 16), (300, 335), (513, 1201),
        (1000, 40)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H", BACK)
def test_backward_matches_64_bits(T, H, dtype, act):
    gate, up, dA = _kept(T, H)
    dA = dA.to(DTYPES[dtype])
    dense = fqt.GatedGrads(dgate=torch.empty_like(dA), dup=torch.empty_like(dA))
    ws = fqt.Workspace.of_size(fqt.fp8_gated_backward_workspace_size(T, H))
    r = fqt.fp8_gated_backward(dA, gate, up, act, out=dense, ws=ws)
    assert r is dense and fqt.sync_status(ws) == 0
    dg, eg, du, eu = _backward64(dA, gate, up, act)
    for got, want, e in ((r.dgate, dg, eg), (r.dup, du, eu)):
        if dtype == "bf16":
            e = e + 2.0 ** -8 * (want.abs() + e)
        assert ((got.double() - want).abs() <= e).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H", BACK)
def test_backward_codes_are_those_of_the_dense_outputs(T, H, dtype, act):
    gate, up, dA = _kept(T, H)
    dA = dA.to(DTYPES[dtype])
    ws = fqt.Workspace.of_size(256)
    r = fqt.fp8_gated_backward(dA, gate, up, act, ws=ws)
    assert fqt.sync_status(ws) == 0 and r.dgate is r.dup is None
    wide = dA.float()  # the same entries: dense outputs in fp32
    dense = fqt.fp8_gated_backward(wide, gate, up, act, out=fqt.GatedGrads(
        dgate=torch.empty_like(wide), dup=torch.empty_like(wide)))
    # a = u act(g) is the gradient of u where a's is u
    a = fqt.fp8_gated_backward(up.dequantize(), gate, up, act,
                               out=fqt.GatedGrads(dup=torch.empty_like(wide))).dup
    _codes_equal(r.qgate, dense.dgate)
    _codes_equal(r.qup, dense.dup)
    _codes_equal(r.qgate_t, dense.dgate.t())
    _codes_equal(r.qup_t, dense.dup.t())
    _codes_equal(r.product_t, a.t())
    # each of them alone
    for name in ("qgate", "qup", "qgate_t", "qup_t", "product_t"):
        ref = getattr(r, name)
        t = fqt.Fp8Tensor.empty(*ref.shape)
        fqt.fp8_gated_backward(dA, gate, up, act, out=fqt.GatedGrads(**{name: t}))
        _same(t, ref)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """Central differences of act(g) u in 64 bits, 2 h = 2^-13 apart: off by h^2 / 6 of the
    third derivative (at most 3 for these) and the roundings of both values."""
    T, H, h = 40, 130, 2.0 ** -14
    gate, up, dA = _kept(T, H)
    gate.codes[gate.codes & 127 == 0] = 0x38  # no zeros: relu has no derivative there
    r = fqt.fp8_gated_backward(dA, gate, up, act, out=fqt.GatedGrads(
        dgate=torch.empty_like(dA), dup=torch.empty_like(dA)))
    g, u, d = gate.dequantize().double(), up.dequantize().double(), dA.double()
    near = g.abs() > h if act == "relu" else torch.ones_like(g).bool()
    f = lambda g, u: _act(g, act)[0] * u  # noqa: E731
    _, eg, _, eu = _backward64(dA, gate, up, act)
    dg = d * (f(g + h, u) - f(g - h, u)) / (2 * h)
    du = d * (f(g, u + h) - f(g, u - h)) / (2 * h)
    off = (d * u).abs() * (h * h / 2 + 2.0 ** -50 * (1 + g.abs()) / h)
    assert ((r.dgate.double() - dg).abs() <= eg + off)[near].all()
    assert ((r.dup.double() - du).abs() <= eu + d.abs() * 2.0 ** -50 * (1 + u.abs()) * (1 + g.abs()) / h).all()


def test_large_and_small_pre_activations():
    """Where sigma is 0, 1 or next to them, and where g^3 passes what fp32 holds."""
    T, H = 8, 256
    vals = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 12.0, -12.0, 88.0, -88.0, 200.0, -200.0, 1e6, -1e6,
                         1e20, -1e20, 1e30, -1e30], device="cuda")
    for v in vals:
        g = torch.full((T, H), float(v), device="cuda")
        gate, up, dA = _f8(g), _f8(torch.ones_like(g)), torch.ones_like(g)
        for act in ACTS:
            r = fqt.fp8_gated_backward(dA, gate, up, act, out=fqt.GatedGrads(
                dgate=torch.empty_like(g), dup=torch.empty_like(g)))
            x = gate.dequantize().double()
            if act == "gelu_tanh" or act == "gelu":
                x = x.clamp(-1e4, 1e4)  # the same limits; 64 bits hold their cubes
            want, slope, _, _ = _act(x, act)
            if float(v) > 1e3:
                want = gate.dequantize().double() if act != "sigmoid" else want
            assert r.dgate.isfinite().all() and r.dup.isfinite().all(), (act, float(v))
            size = 1 + x.abs()
            assert ((r.dgate.double() - slope).abs() <= 1e-5).all(), (act, float(v))
            assert ((r.dup.double() - want).abs() <= 1e-5 * size + 1e-5 * want.abs()).all(), (act, float(v))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H", [(5, 131), (130, 59), (300, 1201)])
def test_backward_rows_of_any_pitch(T, H, dtype):
    """dA and the dense outputs inside wider rows of any alignment; codes between whose
    rows lie other bytes."""
    gate, up, dA = _kept(T, H)
    for t in (gate, up):
        t.codes[:, H:] = 0x7F
        t.scales[:, T:] = 255
    dA = dA.to(DTYPES[dtype])
    ref = fqt.fp8_gated_backward(dA, gate, up, "silu")
    dense = fqt.fp8_gated_backward(dA, gate, up, "silu", out=fqt.GatedGrads(
        dgate=torch.empty_like(dA), dup=torch.empty_like(dA)))
    for gap in (1, 2, 4, 8):
        wide = [torch.full((T + 1, H + gap), 7.0, dtype=dA.dtype, device="cuda") for _ in range(3)]
        wide[0][:T, gap:] = dA
        pitch, pitch_t = -(-H // 16) * 16 + 16, -(-T // 16) * 16 + 16
        raw = [torch.full((n + 1, p), 0x55, dtype=torch.uint8, device="cuda")
               for n, p in ((T, pitch), (T, pitch), (H, pitch_t), (H, pitch_t), (H, pitch_t))]
        qs = [fqt.Fp8Tensor(b[:-1], torch.empty(fqt.Fp8Tensor.scale_shape(n, k), dtype=torch.uint8,
                                                device="cuda"), n, k)
              for b, n, k in zip(raw, (T, T, H, H, H), (H, H, T, T, T))]
        ws = fqt.Workspace.of_size(256)
        fqt.fp8_gated_backward(wide[0][:T, gap:], gate, up, "silu", ws=ws, out=fqt.GatedGrads(
            wide[1][:T, :H], wide[2][:T, gap:], *qs))
        assert fqt.sync_status(ws) == 0
        assert torch.equal(wide[1][:T, :H], dense.dgate)
        assert torch.equal(wide[2][:T, gap:], dense.dup)
        assert (wide[1][T:] == 7).all() and (wide[1][:, H:] == 7).all()
        assert (wide[2][T:] == 7).all() and (wide[2][:, :gap] == 7).all()
        for t, b, name in zip(qs, raw, ("qgate", "qup", "qgate_t", "qup_t", "product_t")):
            _same(t, getattr(ref, name))
            assert (b[-1] == 0x55).all() and (b[:, -(-t.cols // 16) * 16:] == 0x55).all()


def test_backward_entries_that_are_not_finite():
    T, H = 300, 400
    gate, up, dA = _kept(T, H)
    ref = fqt.fp8_gated_backward(dA, gate, up, "silu")
    dA[3, 5], dA[200, 390] = float("nan"), float("inf")
    up.codes[131, 200] = 0x7F
    ws = fqt.Workspace.of_size(256)
    r = fqt.fp8_gated_backward(dA, gate, up, "silu", ws=ws)
    assert fqt.sync_status(ws) == 4
    dense = fqt.fp8_gated_backward(dA, gate, up, "silu", out=fqt.GatedGrads(
        dgate=torch.empty_like(dA), dup=torch.empty_like(dA)), ws=ws)
    assert fqt.sync_status(ws) == 0  # as other dense outputs
    for q, qt, d in ((r.qgate, r.qgate_t, dense.dgate), (r.qup, r.qup_t, dense.dup)):
        fine = d.isfinite()
        zeroed = torch.where(fine, d, torch.zeros_like(d))
        for t, x, f in ((q, zeroed, fine), (qt, zeroed.t(), fine.t())):
            assert torch.equal(t.dequantize()[f], _f8(x).dequantize()[f])
            assert (t.codes[:, :t.cols][~f] & 127 == 127).all()
    fine = torch.ones_like(dA).bool()
    fine[131, 200] = False
    assert (r.product_t.codes[200, 131] & 127) == 127
    keep = fine.t() & (torch.arange(H, device="cuda") != 200)[:, None]
    assert torch.equal(r.product_t.dequantize()[keep], ref.product_t.dequantize()[keep])


# --- two products -----------------------------------------------------------
SUMS = [(1, 1, 1, 1), (1, 1024, 4096, 4096), (2, 131, 1700, 27), (33, 300, 129, 5000),
        (64, 257, 700, 700), (65, 66, 1665, 513), (150, 140, 512, 128), (257, 129, 128, 9000),
        (300, 1201, 335, 335), (2000, 1000, 100, 1300), (3000, 2045, 640, 200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K1,K2", SUMS)
def test_sum_matches_64_bits(M, N, K1, K2, dtype):
    pairs = [(_f8(_randn(M, K, seed=K) * torch.exp(_randn(M, 1, seed=2))),
              _f8(_randn(N, K, seed=K + 1), b)) for K, b in ((K1, 128), (K2, 1))]
    for a, b in pairs:
        for t in (a, b):
            t.codes[:, t.cols:] = 0x7F
            t.scales[t.cols // 512:, :, -(-t.cols // 128) % 4 or 4:] = 255
    want, bound = (x + y for x, y in zip(_sums(*pairs[0]), _sums(*pairs[1])))
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * (want.abs() + bound)
    wide = torch.full((M + 1, N + 3), 7.0, dtype=DTYPES[dtype], device="cuda")
    ws = fqt.Workspace.of_size(fqt.fp8_matmul_sum_workspace_size(M, N, K1, K2))
    fqt.fp8_matmul_sum(*pairs[0], *pairs[1], out=wide[:M, :N], ws=ws)
    assert fqt.sync_status(ws) == 0
    assert ((wide[:M, :N].double() - want).abs() <= bound).all()
    assert (wide[M:] == 7).all() and (wide[:, N:] == 7).all()
    out = fqt.fp8_matmul_sum(*pairs[0], *pairs[1], dtype=DTYPES[dtype])
    assert torch.equal(out, wide[:M, :N])


def test_sum_of_one_product():
    """Pairs without columns, and the same pair twice."""
    a, b = _f8(_randn(100, 300, seed=1)), _f8(_randn(50, 300, seed=2))
    none = lambda n: fqt.Fp8Tensor.empty(n, 0)  # noqa: E731
    ref = fqt.fp8_matmul(a, b)
    assert torch.equal(fqt.fp8_matmul_sum(a, b, none(100), none(50)), ref)
    assert torch.equal(fqt.fp8_matmul_sum(none(100), none(50), a, b), ref)
    out = torch.full((100, 50), 3.0, device="cuda")
    assert (fqt.fp8_matmul_sum(none(100), none(50), none(100), none(50), out=out) == 0).all()
    want, bound = _sums(a, b)
    assert ((fqt.fp8_matmul_sum(a, b, a, b).double() - 2 * want).abs() <= 2 * bound).all()


# --- together ---------------------------------------------------------------
def _step(X, Wg, Wu, W2, dY, act, ws, stream=None):
    """A training step of the block as a user's program runs it."""
    kw = dict(ws=ws, stream=stream)
    qx, qxt = fqt.quantize_fp8(X, cols=True, **kw)
    (qg, qgt), (qu, qut), (q2, q2t) = (fqt.quantize_fp8(w, 128, cols=True, **kw)
                                       for w in (Wg, Wu, W2))
    _, qa, gate, up = fqt.fp8_gated_matmul(qx, qg, qu, act, dense=False, codes=True, keep=True, **kw)
    y = fqt.fp8_matmul(qa, q2, **kw)
    qd, qdt = fqt.quantize_fp8(dY, cols=True, **kw)
    dA = fqt.fp8_matmul(qd, q2t, **kw)
    r = fqt.fp8_gated_backward(dA, gate, up, act, **kw)
    return (y, fqt.fp8_matmul_sum(r.qgate, qgt, r.qup, qut, **kw), fqt.fp8_matmul(r.qgate_t, qxt, **kw),
            fqt.fp8_matmul(r.qup_t, qxt, **kw), fqt.fp8_matmul(qdt, r.product_t, **kw))


def _block(T, D, H):
    return (_randn(T, D, seed=1), *(_randn(H, D, seed=s) / D ** 0.5 for s in (2, 3)),
            _randn(D, H, seed=4) / H ** 0.5, _randn(T, D, seed=5) / T)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,D,H", [(300, 144, 400), (40, 100, 70)])
def test_a_step_matches_the_unquantized_one(T, D, H, act):
    """Every operand is rounded to 3 bits below the leading one, 2.7% in the mean square
    (at most 2^-4), and a gradient passes at most six such roundings, g and u two more:
    15% in the 2-norm, as for the block without a gate.  relu's slope jumps: g's own noise, 2.7%
    sqrt(2) = 3.8% of its size, gives arctan(0.038) / pi = 1.2% of the g another sign, whose
    entries of dg are all wrong, 1.2 of the 50% that are not zero: sqrt(1.2 / 50) = 15.5% more,
    sqrt(0.15^2 + 0.155^2) = 22% together."""
    tensors = _block(T, D, H)
    ws = fqt.Workspace.of_size(1 << 12)
    got = _step(*tensors, act, ws)
    assert fqt.sync_status(ws) == 0
    X, Wg, Wu, W2 = (t.double().requires_grad_() for t in tensors[:4])
    g = X @ Wg.t()
    y = (_act(g, act)[0] * (X @ Wu.t())) @ W2.t()
    ref = (y, *torch.autograd.grad((y * tensors[4].double()).sum(), (X, Wg, Wu, W2)))
    for x, r in zip(got, ref):
        assert (x.double() - r).norm() <= (0.22 if act == "relu" else 0.15) * r.norm()


def test_streams_graphs_and_repeated_calls():
    """The same bits on another stream, again, and from two graphs that share a workspace."""
    tensors = _block(300, 144, 400)
    ws = fqt.Workspace.of_size(1 << 12)
    ref = _step(*tensors, "silu", ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = _step(*tensors, "silu", ws, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, ref))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = _step(*tensors, "silu", ws)
        graphs.append((graph, out))
    for _ in range(2):
        for graph, out in graphs:
            for t in out:
                t.zero_()
            graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
    assert fqt.sync_status(ws) == 0


def test_new_inputs_in_a_graph():
    """A captured call reads its tensors when it is replayed."""
    a, bg, bu = _operands(20, 300, 200)
    out = torch.empty((20, 300), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fqt.fp8_gated_matmul(a, bg, bu, out=out)
    b = _f8(_randn(20, 200, seed=77))
    a.codes.copy_(b.codes), a.scales.copy_(b.scales)
    graph.replay()
    assert torch.equal(out, fqt.fp8_gated_matmul(b, bg, bu)[0])


def test_offsets_past_32_bits():
    """2^20 tokens of 4112 hidden columns, 4.3 GB of codes: the last rows are those of a call on
    them alone (rows of codes and of dense outputs, and the last 128 tokens' columns of a
    transpose, depend on no other rows)."""
    T, H, K, few = 1 << 20, 4112, 64, 256
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    codes = lambda r, c: torch.randint(0, 126, (r, c), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    shape = fqt.Fp8Tensor.scale_shape
    scales = lambda r, c: torch.randint(115, 120, shape(r, c), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    rand = lambda r, c: fqt.Fp8Tensor(codes(r, -(-c // 16) * 16), scales(r, c), r, c)  # noqa: E731
    last = lambda q: fqt.Fp8Tensor(q.codes[T - few:].clone(), q.scales[:, T - few:].contiguous(), few, q.cols)  # noqa: E731
    a, bg, bu = rand(T, K), rand(H, K), rand(H, K)
    out = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    E = fqt.Fp8Tensor.empty
    ws = fqt.Workspace.of_size(256)
    q, gate, up = E(T, H), E(T, H), E(T, H)
    fqt.fp8_gated_matmul(a, bg, bu, "relu", out=out, q=q, gate=gate, up=up, ws=ws)
    _, _, want, bound = _expected(last(a), bg, bu, "relu")
    assert ((out[T - few:].double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all()
    for t, i in ((gate, 0), (up, 1)):
        x, e = _sums(last(a), (bg, bu)[i])
        assert ((last(t).dequantize().double() - x).abs() <= 2.0 ** -4 * x.abs() + 1.07 * e
                + 2.0 ** -10 * x.abs().amax(1, keepdim=True)).all()
    dA = out
    r = fqt.fp8_gated_backward(dA, gate, up, "relu", ws=ws)
    alone = fqt.fp8_gated_backward(dA[T - few:], last(gate), last(up), "relu")
    _same(last(r.qgate), alone.qgate)
    _same(last(r.qup), alone.qup)
    for name in ("qgate_t", "qup_t", "product_t"):
        big, small = getattr(r, name), getattr(alone, name)
        assert torch.equal(big.codes[:, T - few:], small.codes[:, :few])
    del r, q
    dense = fqt.GatedGrads(dgate=torch.empty_like(dA), dup=torch.empty_like(dA))
    fqt.fp8_gated_backward(dA, gate, up, "relu", out=dense, ws=ws)
    small = fqt.fp8_gated_backward(dA[T - few:], last(gate), last(up), "relu", out=fqt.GatedGrads(
        dgate=torch.empty_like(dA[T - few:]), dup=torch.empty_like(dA[T - few:])))
    assert torch.equal(dense.dgate[T - few:], small.dgate)
    assert torch.equal(dense.dup[T - few:], small.dup)
    out = fqt.fp8_matmul_sum(a, bg, a, bu, dtype=torch.bfloat16, ws=ws)
    (x, e), (y, f) = _sums(last(a), bg), _sums(last(a), bu)
    assert ((out[T - few:].double() - x - y).abs() <= (e + f) + 2.0 ** -8 * ((x + y).abs() + e + f)).all()
    assert fqt.sync_status(ws) == 0


def test_gradients_that_are_laid_out_otherwise():
    """A transposed or every other column of a gradient is read as it is."""
    gate, up, dA = _kept(130, 96)
    ref = fqt.fp8_gated_backward(dA, gate, up)
    for x in (dA.t().contiguous().t(), torch.stack([dA, dA], 2).flatten(1)[:, ::2]):
        r = fqt.fp8_gated_backward(x, gate, up)
        _same(r.qgate, ref.qgate), _same(r.qup_t, ref.qup_t)


def test_empty_sizes():
    none, few = fqt.Fp8Tensor.empty(0, 64), _f8(torch.ones((8, 64), device="cuda"))
    assert fqt.fp8_gated_matmul(none, few, few)[0].shape == (0, 8)
    assert fqt.fp8_gated_matmul(few, none, none)[0].shape == (8, 0)
    t = fqt.Fp8Tensor.empty(8, 0)
    out, q, gate, up = fqt.fp8_gated_matmul(t, t, t, "sigmoid", codes=True, keep=True)
    assert (out == 0).all()
    for x in (q, gate, up):
        _codes_equal(x, torch.zeros((8, 8), device="cuda"))
    dA = torch.empty((0, 64), device="cuda")
    r = fqt.fp8_gated_backward(dA, none, none)
    assert r.qgate.shape == (0, 64) and r.product_t.shape == (64, 0)
    assert fqt.fp8_matmul_sum(none, few, none, few).shape == (0, 8)


def test_refusals():
    a, b = _f8(torch.ones((4, 64), device="cuda")), _f8(torch.ones((6, 64), device="cuda"))
    host = fqt.Fp8Tensor.empty(4, 64, device="cpu")
    odd, dA = _f8(torch.ones((6, 65), device="cuda")), torch.ones((4, 64), device="cuda")
    far = fqt.Workspace.of_size(256, "cpu")
    E = fqt.Fp8Tensor.empty
    for bad in (lambda: fqt.fp8_gated_matmul(a, b, odd), lambda: fqt.fp8_gated_matmul(a, odd, b),
                lambda: fqt.fp8_gated_matmul(a, b, a), lambda: fqt.fp8_gated_matmul(a, b, b, "tanh"),
                lambda: fqt.fp8_gated_matmul(host, b, b), lambda: fqt.fp8_gated_matmul(b, host, host),
                lambda: fqt.fp8_gated_matmul(a, b, b, out=dA),
                lambda: fqt.fp8_gated_matmul(a, b, b, q=E(4, 7)),
                lambda: fqt.fp8_gated_matmul(a, b, b, gate=E(6, 4)),
                lambda: fqt.fp8_gated_matmul(a, b, b, up=E(4, 6, device="cpu")),
                lambda: fqt.fp8_gated_matmul(a, b, b, ws=far),
                lambda: fqt.fp8_gated_backward(dA, a, b), lambda: fqt.fp8_gated_backward(dA, b, a),
                lambda: fqt.fp8_gated_backward(dA.cpu(), a, a),
                lambda: fqt.fp8_gated_backward(dA, host, a), lambda: fqt.fp8_gated_backward(dA, a, host),
                lambda: fqt.fp8_gated_backward(dA, a, a, "swish"),
                lambda: fqt.fp8_gated_backward(dA, a, a, out=fqt.GatedGrads(dgate=dA.bfloat16())),
                lambda: fqt.fp8_gated_backward(dA, a, a, out=fqt.GatedGrads(dup=dA.cpu())),
                lambda: fqt.fp8_gated_backward(dA, a, a, out=fqt.GatedGrads(qgate_t=E(4, 64))),
                lambda: fqt.fp8_gated_backward(dA, a, a, out=fqt.GatedGrads(qup=E(64, 4))),
                lambda: fqt.fp8_gated_backward(dA, a, a, ws=far),
                lambda: fqt.fp8_matmul_sum(a, b, a, odd), lambda: fqt.fp8_matmul_sum(a, b, b, a),
                lambda: fqt.fp8_matmul_sum(a, a, host, a), lambda: fqt.fp8_matmul_sum(a, b, a, b, ws=far),
                lambda: fqt.fp8_matmul_sum(a, b, a, b, out=dA)):
        with pytest.raises(ValueError):
            bad()
    q, q64 = E(4, 6), torch.empty_like(dA)
    for bad in (lambda: fqt.fp8_gated_matmul(a, b, b, dense=False),
                lambda: fqt.fp8_gated_matmul(a, b, b, gate=q, up=q),
                lambda: fqt.fp8_gated_backward(dA, a, a, out=fqt.GatedGrads()),
                lambda: fqt.fp8_gated_backward(dA, a, a, out=fqt.GatedGrads(dgate=q64, dup=q64)),
                lambda: fqt.fp8_gated_matmul(a, b, b, ws=fqt.Workspace.of_size(128))):
        with pytest.raises(fqt.FqtError):
            bad()
    with pytest.raises(TypeError):
        fqt.fp8_gated_matmul(a, b, b, dtype=torch.float16)
    with pytest.raises(TypeError):
        fqt.fp8_gated_backward(dA.half(), a, a)
