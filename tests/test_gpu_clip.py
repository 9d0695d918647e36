"""The global norm of a list of gradients, and clipping, against 64 bits.

Tolerances.  Squares are added in fp32 over the at most 8 x 8 entries that a thread
takes of a unit, then in float-float and in 64 bits: the sum of squares is off by at
most 64 x 2^-24 of itself, the norm by half of that, 2e-6, and its rounding to fp32
adds 6e-8: 2.1e-6.  The factor inherits that and each entry one rounding of its type.
"""
import math

import pytest
import torch

from paper_2010_14298_gb300 import fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
REL = 2.1e-6


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _grads(counts, dtypes, seed=0, scale=1.0, offset=0):
    """Tensors `offset` entries into their memory."""
    g = _gen(seed)
    out = []
    for i, n in enumerate(counts):
        t = torch.randn(n + offset, generator=g, device="cuda") * scale * (1 + i % 5)
        out.append(t.to(dtypes[i % len(dtypes)])[offset:])
    return out


def _norm64(grads):
    return math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))


def _check(grads, max_norm, out, norm):
    want = _norm64(grads)
    assert abs(float(norm) - want) <= REL * want
    f = max_norm / want if want > max_norm else 1.0
    for g, o in zip(grads, out):
        ref = g.double() * f
        if f == 1.0:
            assert torch.equal(o, g)
        else:
            assert ((o.double() - ref).abs() <= (1.1 * ROUND[g.dtype] + REL) * ref.abs()
                    + 1e-45).all()


LISTS = [[1], [7, 1, 3], [4096, 1, 8191, 8192, 8193, 16384, 16385], [100000], [3] * 41, [17] * 251,
         [5] * 1021, [1, 300000, 2] * 700, [5_000_000, 64, 64, 250_001]]
F32, BF16 = [torch.float32], [torch.bfloat16]
MIXED = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtypes", [F32, BF16, MIXED], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("counts", LISTS, ids=lambda c: f"{len(c)}x{max(c)}")
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_matches_64_bits(counts, dtypes, max_norm):
    if sum(counts) > 10 ** 8:
        counts = counts[:200]
    grads = _grads(counts, dtypes)
    out = [torch.full_like(g, 7.0) for g in grads]
    ws = fqt.Workspace.of_size(fqt.clip_grad_norm_workspace_size(grads))
    norm = fqt.clip_grad_norm(grads, max_norm, out=out, ws=ws)
    assert fqt.sync_status(ws) == 0
    _check(grads, max_norm, out, norm)
    assert float(fqt.grad_norm(grads, ws=ws)) == float(norm)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("a,b", [(0, 0), (1, 1), (3, 3), (0, 1), (2, 0), (5, 7)])
def test_any_alignment(a, b, dtype):
    """Inputs and outputs at any entry of 16 bytes, alike or not; nothing beside
    them is written."""
    n = 40003
    grads = _grads([n, 13], [dtype], offset=a)
    mem = [torch.full((n + 32,), 9.0, device="cuda").to(dtype) for _ in grads]
    out = [m[16 + b:16 + b + g.numel()] for m, g in zip(mem, grads)]
    norm = fqt.clip_grad_norm(grads, 1.0, out=out)
    _check(grads, 1.0, out, norm)
    for m, o in zip(mem, out):
        assert (m[:16 + b] == 9).all() and (m[16 + b + o.numel():] == 9).all()


def test_in_place():
    grads = _grads([70001, 5, 12], MIXED)
    before = [g.clone() for g in grads]
    norm = fqt.clip_grad_norm(grads, 2.0)
    _check(before, 2.0, grads, norm)
    kept = [g.clone() for g in grads]
    fqt.clip_grad_norm(fqt.TensorList(grads), 1e9)
    assert all(torch.equal(a, b) for a, b in zip(kept, grads))


@pytest.mark.parametrize("scale", [1e-44, 1e-40, 1e-30, 1e-20, 1e15, 1e25, 1e38])
def test_squares_outside_fp32(scale):
    """Entries whose squares fp32 cannot hold."""
    x = torch.linspace(0.1, 1.0, 5000, device="cuda") * scale
    grads = [x, torch.zeros(300, device="cuda"), x[:7].clone()]
    want = _norm64(grads)
    got = float(fqt.grad_norm(grads))
    if want < 3e38:
        assert abs(got - want) <= REL * want + 1.5e-45
    else:
        assert got == math.inf
    out = [torch.empty_like(g) for g in grads]
    fqt.clip_grad_norm(grads, want / 4, out=out)
    if 1e-35 < want < 1e38:  # a quarter of entries that are no subnormals
        for g, o in zip(grads, out):
            assert ((o.double() - g.double() / 4).abs() <= 3e-6 * g.double().abs()).all()


def test_large_and_tiny_together():
    grads = [torch.full((1000,), 1e-30, device="cuda"), torch.full((3,), 2.0, device="cuda"),
             torch.full((9,), 1e22, device="cuda")]
    assert abs(float(fqt.grad_norm(grads)) / 3e22 - 1) <= REL


def test_zeros_and_a_largest_norm_of_zero():
    z = [torch.zeros(1000, device="cuda"), torch.zeros(3, device="cuda")]
    assert float(fqt.clip_grad_norm(z, 1.0)) == 0.0 and (z[0] == 0).all()
    g = _grads([500], F32)
    fqt.clip_grad_norm(g, 0.0)
    assert (g[0] == 0).all()


def test_empty_tensors_in_the_list():
    e = torch.empty(0, device="cuda")
    grads = [e, torch.full((4,), 2.0, device="cuda"), e.clone(), e.bfloat16()]
    assert float(fqt.clip_grad_norm(grads, 2.0)) == 4.0
    assert (grads[1] == 1.0).all()
    assert float(fqt.grad_norm([e, e])) == 0.0
    assert float(fqt.clip_grad_norm([e] * 5, 1.0)) == 0.0


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_changes_nothing(value):
    grads = _grads([9000, 20], MIXED)
    grads[1][11] = value
    before = [g.clone() for g in grads]
    ws = fqt.Workspace.of_size(fqt.clip_grad_norm_workspace_size(grads))
    norm = float(fqt.clip_grad_norm(grads, 1.0, ws=ws))
    assert math.isnan(norm) if math.isnan(value) else norm == math.inf
    assert fqt.sync_status(ws) == 4 and fqt.sync_status(ws) == 0
    for a, b in zip(before, grads):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_the_same_bits_again_another_stream_and_graphs():
    grads = fqt.TensorList(_grads([1_000_003, 77, 64, 300_000], F32))
    mem = [torch.zeros_like(g) for g in grads]
    out = fqt.TensorList(mem)
    ws = fqt.Workspace.of_size(fqt.clip_grad_norm_workspace_size(grads))
    norm = fqt.clip_grad_norm(grads, 1.0, out=out, ws=ws).clone()
    want = [o.clone() for o in out]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    again = fqt.clip_grad_norm(grads, 1.0, out=out, ws=ws, stream=s)
    s.synchronize()
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fqt.clip_grad_norm(grads, 1.0, out=out, norm=again, ws=ws)
    for o in mem:
        o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    g = [torch.ones(8, device="cuda")]
    for bad in (lambda: fqt.clip_grad_norm([], 1.0),
                lambda: fqt.clip_grad_norm([g[0].cpu()], 1.0),
                lambda: fqt.clip_grad_norm([torch.ones((4, 4), device="cuda").t()[:3]], 1.0),
                lambda: fqt.clip_grad_norm(g, 1.0, out=[torch.ones(7, device="cuda")]),
                lambda: fqt.clip_grad_norm(g, 1.0, out=[g[0].bfloat16()]),
                lambda: fqt.clip_grad_norm(g, 1.0, norm=torch.ones(2, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        fqt.clip_grad_norm([g[0].half()], 1.0)
    for m in (-1.0, float("nan")):
        with pytest.raises(fqt.FqtError) as e:
            fqt.clip_grad_norm(g, m)
        assert e.value.status == 1
    with pytest.raises(fqt.FqtError) as e:
        fqt.clip_grad_norm(g, 1.0, ws=fqt.Workspace.of_size(64))
    assert e.value.status == 6
