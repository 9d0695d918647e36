"""The global norm and clipping at the ends of fp32's range and over long lists.

Tolerances.  A thread adds the squares of a unit, at most 64 + 1 of them, in fp32, and
everything after that in pairs of fp32: the sum of squares is off by at most 65 x 2^-24
of itself, the norm by half of that, 2e-6, and its rounding to fp32 adds 6e-8: 2.1e-6.
The factor inherits that, and an entry adds a rounding of the factor, one of the product
and one of its type.
"""
import math

import pytest
import torch

from paper_2010_14298_gb300 import fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
REL = 2.1e-6


@pytest.mark.parametrize("dtype,count,value", [(torch.float32, 5 << 28, 2.0 ** 49),
                                               (torch.bfloat16, 6 << 29, 3.6e14)],
                         ids=["f32", "bf16"])
def test_many_large_entries(dtype, count, value):
    """Squares of 2^98 that fp32 holds one by one, and not their sum: the norm is about
    2^64, and the list is clipped."""
    g = torch.full((count,), value, dtype=dtype, device="cuda")
    value = float(g[0])
    want = math.sqrt(count) * value
    ws = fqt.Workspace.of_size(fqt.clip_grad_norm_workspace_size([g]))
    norm = fqt.clip_grad_norm([g], 1.0, ws=ws)
    assert fqt.sync_status(ws) == 0
    assert abs(float(norm) / want - 1) <= REL
    for end in (float(g.min()), float(g.max())):
        assert abs(end / (value / want) - 1) <= REL + 3 * 2.0 ** -24 + ROUND[dtype]


@pytest.mark.parametrize("value", [1.1e-38, 1.1e-20, 1.3e-16, 0.7, 1.1e13, 1.1e20, 1.1e30])
def test_long_lists_of_equal_entries(value):
    """2^32 entries of any size: the sums of those whose squares fp32 does not hold keep
    as many bits as the others'."""
    t = torch.full((1 << 26,), value, device="cuda")
    grads = fqt.TensorList([t] * 64)
    want = math.sqrt(float(1 << 32)) * float(t[0].double())
    assert abs(float(fqt.grad_norm(grads)) / want - 1) <= REL


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1e30, 1.0, 1e-3, 1e-30])
@pytest.mark.parametrize("top", [1e37, 3e38])
def test_factors_that_fp32_does_not_hold(top, max_norm, dtype):
    """max_norm / norm under fp32's normal numbers, or under all of them: the entries,
    which are no larger than the norm, are still rounded once.  A norm past fp32 is
    written as infinity, and is no entry that is not finite."""
    grads = [(torch.linspace(0.1, 1.0, n, device="cuda") * top).to(dtype) for n in (40003, 7, 512)]
    want = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))
    out = [torch.full_like(g, 7.0) for g in grads]
    ws = fqt.Workspace.of_size(fqt.clip_grad_norm_workspace_size(grads))
    norm = float(fqt.clip_grad_norm(grads, max_norm, out=out, ws=ws))
    assert fqt.sync_status(ws) == 0
    assert norm == math.inf if want > 3.5e38 else abs(norm / want - 1) <= REL
    for g, o in zip(grads, out):
        ref = g.double() * (max_norm / want)
        tol = (REL + 3 * 2.0 ** -24 + ROUND[dtype]) * ref.abs()
        assert ((o.double() - ref).abs() <= tol).all()


@pytest.mark.parametrize("counts", [[64, 3, 100_000] * 700, [5] * 1021, [1 << 20] * 90],
                         ids=["2100", "1021", "90"])
def test_in_place_as_into_other_tensors(counts):
    """The same bits, over more tensors than one launch takes too, and none changed where
    the norm is small enough."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    grads = [torch.randn(n, generator=gen, device="cuda").to(
        torch.bfloat16 if i % 3 == 0 else torch.float32) for i, n in enumerate(counts)]
    before = [g.clone() for g in grads]
    want = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))
    out = [torch.full_like(g, 7.0) for g in grads]
    apart = fqt.clip_grad_norm(grads, want / 3, out=out)
    norm = fqt.clip_grad_norm(grads, want / 3)
    assert torch.equal(norm, apart) and abs(float(norm) / want - 1) <= REL
    for g, o, b in zip(grads, out, before):
        assert torch.equal(g, o)
        ref = b.double() / 3
        assert ((g.double() - ref).abs()
                <= (REL + 3 * 2.0 ** -24 + ROUND[g.dtype]) * ref.abs()).all()
    fqt.clip_grad_norm(grads, want)
    assert all(torch.equal(g, o) for g, o in zip(grads, out))
