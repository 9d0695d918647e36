"""The gated feed-forward block's C entry points refuse bad requests before any CUDA call,
and both marshallings of the binding take and refuse the same (no GPU needed)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2010_14298_gb300 import fqt  # noqa: E402

EINVAL, EWORKSPACE = 1, 6
RAW = torch.zeros((1 << 17) + 256, dtype=torch.uint8)
P = (RAW.data_ptr() + 255) & ~255


def _at(k):
    """A place of its own for each k."""
    return P + 4096 * k


def _f8(rows, cols, k=0, pitch=None, block_rows=1, codes=None, scales=None):
    return fqt._F8(rows, cols, -(-cols // 16) * 16 if pitch is None else pitch, block_rows, 0,
                   _at(k) if codes is None else codes, _at(k) + 2048 if scales is None else scales)


def _ref(q):
    return ctypes.byref(q) if q is not None else None


BAD_CODES = [dict(pitch=48), dict(pitch=72), dict(pitch=1 << 40), dict(codes=_at(9) + 8),
             dict(codes=0), dict(scales=0), dict(scales=_at(9) + 4)]


def _gated(A=None, Bg=None, Bu=None, act=0, dtype=0, out=_at(5), ldo=20, q=None, gate=None,
           up=None, ws=_at(6), nbytes=256):
    A, Bg, Bu = A or _f8(10, 64, 0), Bg or _f8(20, 64, 1), Bu or _f8(20, 64, 2)
    return fqt.load().fqt_fp8_gated_matmul(_ref(A), _ref(Bg), _ref(Bu), act, dtype, out, ldo,
                                           _ref(q), _ref(gate), _ref(up), ws, nbytes, None)


def test_forward_refusals():
    lib = fqt.load()
    none = ctypes.POINTER(fqt._F8)()
    q = _f8(10, 64)
    for a in ((none, q, q), (q, none, q), (q, q, none)):
        assert lib.fqt_fp8_gated_matmul(*a, 0, 0, _at(5), 64, none, none, none, _at(6), 256,
                                        None) == EINVAL
    assert _gated(act=5) == EINVAL and _gated(act=-1) == EINVAL and _gated(dtype=2) == EINVAL
    assert _gated(out=None) == EINVAL  # nothing asked for
    assert _gated(Bg=_f8(20, 65, 1)) == EINVAL and _gated(Bu=_f8(20, 63, 2)) == EINVAL
    assert _gated(Bu=_f8(21, 64, 2)) == EINVAL
    assert _gated(A=_f8(-1, 64)) == EINVAL and _gated(A=_f8((1 << 22) + 1, 64)) == EINVAL
    assert _gated(Bu=_f8(20, 64, 2, block_rows=64)) == EINVAL
    assert _gated(ldo=19) == EINVAL and _gated(ldo=1 << 41) == EINVAL
    assert _gated(out=_at(5) + 2) == EINVAL and _gated(out=_at(5) + 1, dtype=1) == EINVAL
    for bad in BAD_CODES:
        for name, rows in (("A", 10), ("Bg", 20), ("Bu", 20)):
            assert _gated(**{name: _f8(rows, 64, 9, **bad)}) == EINVAL, (name, bad)
        # an output's sizes are the call's: 20 columns
        bad = dict(bad, pitch=16) if bad.get("pitch") == 48 else bad
        for name in ("q", "gate", "up"):
            assert _gated(**{name: _f8(10, 20, 9, **bad)}) == EINVAL, (name, bad)
    # two outputs in one place
    assert _gated(q=_f8(10, 20, 7), gate=_f8(10, 20, 7)) == EINVAL
    assert _gated(gate=_f8(10, 20, 7), up=_f8(10, 20, 8, codes=_at(7))) == EINVAL
    assert _gated(gate=_f8(10, 20, 7), up=_f8(10, 20, 8, scales=_at(7) + 2048)) == EINVAL
    # an output where an operand is
    for k in range(3):
        for name in ("q", "gate", "up"):
            assert _gated(**{name: _f8(10, 20, 7, codes=_at(k))}) == EINVAL, (name, k)
            assert _gated(**{name: _f8(10, 20, 7, scales=_at(k) + 2048)}) == EINVAL, (name, k)
        assert _gated(out=_at(k)) == EINVAL
    assert _gated(ws=None) == EWORKSPACE and _gated(nbytes=128) == EWORKSPACE
    assert _gated(ws=_at(6) + 16) == EWORKSPACE
    # nothing to do: the sizes of the outputs are set
    q = _f8(3, 3, 7)
    assert _gated(A=_f8(0, 64), q=q, ws=None) == 0 and (q.rows, q.cols, q.block_rows) == (0, 20, 1)
    assert _gated(Bg=_f8(0, 64, 1), Bu=_f8(0, 64, 2), out=None, q=q) == 0


def _back(dA=_at(0), ldda=64, dtype=0, gate=None, up=None, act=0, dgate=_at(3), lddg=64,
          dup=_at(4), lddu=64, q=(None,) * 5, ws=_at(12), nbytes=256):
    gate, up = gate or _f8(4, 64, 1), up or _f8(4, 64, 2)
    return fqt.load().fqt_fp8_gated_backward(dA, ldda, dtype, _ref(gate), _ref(up), act, dgate, lddg,
                                             dup, lddu, *map(_ref, q), ws, nbytes, None)


def test_backward_refusals():
    lib = fqt.load()
    none = ctypes.POINTER(fqt._F8)()
    q = _f8(4, 64)
    for a in ((none, q), (q, none)):
        assert lib.fqt_fp8_gated_backward(_at(0), 64, 0, *a, 0, _at(3), 64, None, 64, none, none, none,
                                          none, none, _at(12), 256, None) == EINVAL
    assert _back(act=5) == EINVAL and _back(act=-1) == EINVAL and _back(dtype=2) == EINVAL
    assert _back(dgate=None, dup=None) == EINVAL  # nothing asked for
    assert _back(dA=None) == EINVAL and _back(dA=_at(0) + 2) == EINVAL
    assert _back(ldda=63) == EINVAL and _back(ldda=1 << 41) == EINVAL
    assert _back(lddg=63) == EINVAL and _back(lddu=63) == EINVAL and _back(lddu=1 << 41) == EINVAL
    assert _back(dgate=_at(3) + 2) == EINVAL and _back(dup=_at(4) + 1, dtype=1) == EINVAL
    assert _back(dgate=_at(3), dup=_at(3)) == EINVAL
    assert _back(up=_f8(4, 65, 2)) == EINVAL and _back(up=_f8(5, 64, 2)) == EINVAL
    assert _back(gate=_f8(4, 0, 1), up=_f8(4, 0, 2)) == EINVAL
    assert _back(gate=_f8(-1, 64, 1), up=_f8(-1, 64, 2)) == EINVAL
    far = 1 << 22
    assert _back(gate=_f8(far + 1, 64, 1), up=_f8(far + 1, 64, 2)) == EINVAL
    assert _back(gate=_f8(4, 64, 1, block_rows=3)) == EINVAL
    for bad in BAD_CODES:
        assert _back(gate=_f8(4, 64, 9, **bad)) == EINVAL and _back(up=_f8(4, 64, 9, **bad)) == EINVAL
        for i in range(5):  # the transposes have 4 columns
            b = dict(bad, pitch=0) if i > 1 and bad.get("pitch") == 48 else bad
            q = [None] * 5
            q[i] = _f8(0, 0, 9, **{"pitch": 64, **b})
            assert _back(q=q) == EINVAL, (i, bad)
    for i, j in ((0, 1), (0, 2), (2, 3), (3, 4)):
        q = [None] * 5
        q[i], q[j] = _f8(0, 0, 7, pitch=64), _f8(0, 0, 7, pitch=64)
        assert _back(q=q) == EINVAL
    # an output where dA, g or u are
    assert _back(dgate=_at(0)) == EINVAL and _back(dup=_at(0)) == EINVAL
    for i in range(5):
        for k in (1, 2):
            for place in (dict(codes=_at(k)), dict(scales=_at(k) + 2048)):
                q = [None] * 5
                q[i] = _f8(0, 0, 7, pitch=64, **place)
                assert _back(q=q) == EINVAL, (i, k)
    assert _back(ws=None) == EWORKSPACE and _back(nbytes=16) == EWORKSPACE
    assert _back(ws=_at(12) + 8) == EWORKSPACE
    q = [_f8(9, 9, i) for i in range(5)]
    assert _back(gate=_f8(0, 64, 1), up=_f8(0, 64, 2), dA=None, q=q, ws=None) == 0
    assert [(x.rows, x.cols) for x in q] == [(0, 64)] * 2 + [(64, 0)] * 3


def _sum(A1=None, B1=None, A2=None, B2=None, dtype=0, out=_at(5), ldo=20, ws=_at(6), nbytes=256):
    args = A1 or _f8(10, 64, 0), B1 or _f8(20, 64, 1), A2 or _f8(10, 32, 2), B2 or _f8(20, 32, 3)
    return fqt.load().fqt_fp8_matmul_sum(*map(_ref, args), dtype, out, ldo, ws, nbytes, None)


def test_sum_refusals():
    lib = fqt.load()
    none = ctypes.POINTER(fqt._F8)()
    q = _f8(10, 64)
    for i in range(4):
        a = [q] * 4
        a[i] = none
        assert lib.fqt_fp8_matmul_sum(*a, 0, _at(5), 64, _at(6), 256, None) == EINVAL
    assert _sum(dtype=2) == EINVAL and _sum(out=None) == EINVAL and _sum(out=_at(5) + 2) == EINVAL
    assert _sum(ldo=19) == EINVAL and _sum(ldo=1 << 41) == EINVAL
    assert _sum(A1=_f8(10, 65)) == EINVAL and _sum(B2=_f8(20, 33, 3)) == EINVAL
    assert _sum(A2=_f8(11, 32, 2)) == EINVAL and _sum(B2=_f8(21, 32, 3)) == EINVAL
    assert _sum(A2=_f8(10, 32, 2, block_rows=2)) == EINVAL
    assert _sum(A1=_f8(-1, 64), A2=_f8(-1, 32, 2)) == EINVAL
    far = (1 << 22) + 1
    assert _sum(A1=_f8(far, 64), A2=_f8(far, 32, 2)) == EINVAL
    for bad in BAD_CODES:
        for name, rows, cols in (("A1", 10, 64), ("B1", 20, 64), ("A2", 10, 64), ("B2", 20, 64)):
            kw = {name: _f8(rows, cols, 9, **bad)}
            if name[1] == "2":
                kw.setdefault("A2", _f8(10, 64, 2)), kw.setdefault("B2", _f8(20, 64, 3))
            assert _sum(**kw) == EINVAL, (name, bad)
    assert _sum(ws=None) == EWORKSPACE and _sum(nbytes=16) == EWORKSPACE
    assert _sum(ws=_at(6) + 16) == EWORKSPACE
    assert _sum(A1=_f8(0, 64), A2=_f8(0, 32, 2)) == 0 and _sum(B1=_f8(0, 64, 1), B2=_f8(0, 32, 3)) == 0


@pytest.mark.parametrize("calls", ["extension", "ctypes"])
def test_both_marshallings_take_and_refuse_the_same(calls):
    n = fqt.native() if calls == "extension" else fqt._CtypesCalls(fqt.load())
    E = lambda r, c: fqt.Fp8Tensor.empty(r, c, device="cpu")  # noqa: E731
    a, b, odd, none = E(4, 64), E(6, 64), E(6, 65), E(0, 64)
    X, ws = torch.zeros(8, 64), torch.zeros(512, dtype=torch.uint8)
    assert n.fp8_gated_matmul(a, b, odd, 0, 0, X, 6, None, None, None, ws, 512, 0) == EINVAL
    assert n.fp8_gated_matmul(a, b, b, 9, 0, X, 6, None, None, None, ws, 512, 0) == EINVAL
    assert n.fp8_gated_matmul(a, b, b, 0, 0, None, 6, None, None, None, ws, 512, 0) == EINVAL
    assert n.fp8_gated_matmul(none, b, b, 0, 0, None, 6, E(0, 6), None, E(0, 6), ws, 512, 0) == 0
    back = lambda *q: n.fp8_gated_backward(X, 64, 0, a, a, 0, None, 64, None, 64, *q, ws, 512, 0)  # noqa: E731
    assert back(None, None, None, None, None) == EINVAL
    assert n.fp8_gated_backward(X, 64, 0, a, b, 0, X, 64, None, 64, *(None,) * 5, ws, 512, 0) == EINVAL
    assert n.fp8_gated_backward(X, 64, 0, none, none, 0, None, 64, None, 64, None, E(0, 64), None,
                                E(64, 0), E(64, 0), ws, 512, 0) == 0
    assert n.fp8_matmul_sum(a, b, a, odd, 0, X, 6, ws, 512, 0) == EINVAL
    assert n.fp8_matmul_sum(none, b, none, b, 0, X, 6, ws, 512, 0) == 0
    with pytest.raises((TypeError, ValueError)):
        fqt.fp8_gated_matmul(a, b, b, "swish")
    for call in (lambda: fqt.fp8_gated_matmul(a, b, b), lambda: fqt.fp8_matmul_sum(a, b, a, b),
                 lambda: fqt.fp8_gated_backward(X, a, a)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()
