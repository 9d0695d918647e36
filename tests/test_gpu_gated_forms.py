"""The gated block's operators in forms that its other tests leave out: blocks of one row
where weights mostly have 128 x 128 and the other way round, outputs between one another's
rows, two streams at once, the same bits again at the size of a prompt.  Tolerances as in
test_gpu_gated.py."""
import pytest
import torch

from paper_2010_14298_gb300 import fqt
from test_gpu_gated import (ACTS, DTYPES, _backward64, _codes_equal, _expected, _f8, _kept, _randn,
                            _same, _step, _sums)

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


@pytest.mark.parametrize("blocks", [(128, 1, 1), (128, 128, 128), (1, 1, 128), (1, 128, 1)])
@pytest.mark.parametrize("T,H,K", [(3, 300, 700), (50, 130, 1300), (300, 335, 1201), (2100, 1000, 200)])
def test_forward_blocks_of_either_kind(T, H, K, blocks):
    """Rows of very different sizes, so that a scale taken from another row would show."""
    ba, bg, bu = blocks
    size = lambda n, s: torch.exp(2 * _randn(n, 1, seed=s))  # noqa: E731
    a = _f8(_randn(T, K, seed=1) * size(T, 2), ba)
    wg, wu = (_f8(_randn(H, K, seed=s) * size(H, s + 4) / K ** 0.5, b) for s, b in ((3, bg), (4, bu)))
    assert (a.block_rows, wg.block_rows, wu.block_rows) == blocks
    ws = fqt.Workspace.of_size(256)
    for act in ("silu", "gelu"):
        _, _, want, bound = _expected(a, wg, wu, act)
        for dtype in DTYPES.values():
            e = bound + (2.0 ** -8 * (want.abs() + bound) if dtype is torch.bfloat16 else 0)
            out, q, _, _ = fqt.fp8_gated_matmul(a, wg, wu, act, dtype=dtype, codes=True, ws=ws)
            assert ((out.double() - want).abs() <= e).all(), act
            alone = fqt.fp8_gated_matmul(a, wg, wu, act, dtype=dtype, ws=ws)[0]
            assert ((alone.double() - want).abs() <= e).all(), act
            assert q.block_rows == 1
            if dtype is torch.float32:
                _codes_equal(q, out)
    assert fqt.sync_status(ws) == 0


def _wide64(dA, gate, up, act):
    """_backward64 for checkpoints far from zero.  Its s (1 - s) of sigmoid is off by 2^-53 e^g
    of itself in 64 bits (1 - s is rounded at 2^-53, and is e^-g): more than a kernel's
    (24 + 10 g) 2^-24 from g = 26 on.  Here 1 - s is sigma(-g)."""
    dg, eg, du, eu = _backward64(dA, gate, up, act)
    if act == "sigmoid":
        g = gate.dequantize().double()
        d = dA.double() * up.dequantize().double()
        slope = torch.sigmoid(g) * torch.sigmoid(-g)
        dg = d * slope
        eg = d.abs() * ((24 + 10 * g.abs()) * slope * 2.0 ** -24 + 2.0 ** -120) + 2.0 ** -22 * dg.abs() + 2.0 ** -120
    return dg, eg, du, eu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("blocks", [(128, 128), (128, 1), (1, 128)])
@pytest.mark.parametrize("T,H", [(1, 130), (64, 128), (300, 335), (513, 1201)])
def test_backward_from_checkpoints_of_either_kind(T, H, blocks, dtype):
    g, u, dA = _kept(T, H)
    size = torch.exp(_randn(T, 1, seed=12))
    gate, up = (_f8(t.dequantize() * size, b) for t, b in zip((g, u), blocks))
    dA = dA.to(DTYPES[dtype])
    ws = fqt.Workspace.of_size(256)
    for act in ACTS:
        dense = fqt.GatedGrads(dgate=torch.empty_like(dA), dup=torch.empty_like(dA))
        r = fqt.fp8_gated_backward(dA, gate, up, act, out=dense, ws=ws)
        dg, eg, du, eu = _wide64(dA, gate, up, act)
        for got, want, e in ((r.dgate, dg, eg), (r.dup, du, eu)):
            if dtype == "bf16":
                e = e + 2.0 ** -8 * (want.abs() + e)
            assert ((got.double() - want).abs() <= e).all(), act
        codes = fqt.fp8_gated_backward(dA, gate, up, act, ws=ws)
        wide = dA.float()
        dense = fqt.fp8_gated_backward(wide, gate, up, act, ws=ws, out=fqt.GatedGrads(
            dgate=torch.empty_like(wide), dup=torch.empty_like(wide)))
        _codes_equal(codes.qgate, dense.dgate), _codes_equal(codes.qup, dense.dup)
        _codes_equal(codes.qgate_t, dense.dgate.t()), _codes_equal(codes.qup_t, dense.dup.t())
    assert fqt.sync_status(ws) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H", [(5, 131), (300, 400), (700, 1000)])
def test_both_gradients_in_one_buffer(T, H, dtype):
    """dg and du as halves of one gradient, as one product of a shared weight reads them."""
    gate, up, dA = _kept(T, H)
    dA = dA.to(DTYPES[dtype])
    ref = fqt.fp8_gated_backward(dA, gate, up, out=fqt.GatedGrads(
        dgate=torch.empty_like(dA), dup=torch.empty_like(dA)))
    both = torch.empty((T, 2 * H), dtype=dA.dtype, device="cuda")
    for codes in (False, True):
        both.fill_(7.0)
        out = fqt.GatedGrads.empty(T, H) if codes else fqt.GatedGrads()
        out.dgate, out.dup = both[:, :H], both[:, H:]
        fqt.fp8_gated_backward(dA, gate, up, out=out)
        assert torch.equal(both, torch.cat([ref.dgate, ref.dup], 1))
    with pytest.raises(fqt.FqtError):
        fqt.fp8_gated_backward(dA, gate, up, out=fqt.GatedGrads(dgate=both[:, :H],
                                                                dup=both[:, H - 1:2 * H - 1]))


def _block(T, D, H, seed):
    return (_randn(T, D, seed=seed), *(_randn(H, D, seed=seed + s) / D ** 0.5 for s in (1, 2)),
            _randn(D, H, seed=seed + 3) / H ** 0.5, _randn(T, D, seed=seed + 4) / T)


def test_two_streams_at_once():
    """Two steps of their own sizes on two streams, a workspace each, give the bits that each
    gives alone."""
    blocks = [_block(1500, 336, 1200, 20), _block(40, 1024, 1000, 30)]
    works = [fqt.Workspace.of_size(1 << 12) for _ in blocks]
    refs = [_step(*b, "silu", ws) for b, ws in zip(blocks, works)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = []
    for _ in range(5):
        for b, ws, s in zip(blocks, works, streams):
            got.append(_step(*b, "silu", ws, stream=s))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert all(torch.equal(x, y) for x, y in zip(out, refs[i % 2]))
    assert all(fqt.sync_status(ws) == 0 for ws in works)


def test_the_same_bits_again_at_8192_tokens():
    """The forward's and the backward's codes, and what is made of them, twenty times over."""
    block = _block(8192, 512, 2048, 40)
    ws = fqt.Workspace.of_size(1 << 12)
    ref = _step(*block, "silu", ws)
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    for i in range(20):
        flush.fill_(i)
        assert all(torch.equal(x, y) for x, y in zip(_step(*block, "silu", ws), ref))
    assert fqt.sync_status(ws) == 0


def test_sum_of_blocks_of_either_kind():
    for ba, bb in ((128, 1), (128, 128), (1, 1)):
        for M, N, K1, K2 in ((3, 300, 700, 129), (300, 1201, 335, 40), (2100, 1000, 200, 200)):
            size = torch.exp(2 * _randn(M, 1, seed=2))
            pairs = [(_f8(_randn(M, K, seed=K) * size, ba),
                      _f8(_randn(N, K, seed=K + 1) * torch.exp(_randn(N, 1, seed=3)), bb))
                     for K in (K1, K2)]
            want, bound = (x + y for x, y in zip(_sums(*pairs[0]), _sums(*pairs[1])))
            out = fqt.fp8_matmul_sum(*pairs[0], *pairs[1])
            assert ((out.double() - want).abs() <= bound).all()


def test_codes_beside_either_kind_of_weights():
    """The kind of an operand's blocks decides nothing but its scales: weights whose rows all
    have one scale give the same bits with blocks of one row."""
    w = [torch.randint(-4, 5, (300, 400), device="cuda").float() for _ in range(2)]
    for x in w:
        x[:, ::128] = 4.0  # (every row's blocks have their tile's largest entry)
    a = _f8(_randn(200, 400, seed=5))
    one, tile = ([_f8(x, b) for x in w] for b in (1, 128))
    for x, y in zip(one, tile):
        _same(x, y)
    got, ref = (fqt.fp8_gated_matmul(a, *k, codes=True, keep=True) for k in (one, tile))
    assert torch.equal(got[0], ref[0])
    for x, y in zip(got[1:], ref[1:]):
        _same(x, y)
