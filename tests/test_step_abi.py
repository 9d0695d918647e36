"""The C entry points around the quantized layers refuse bad requests before any
CUDA call (no GPU needed)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2010_14298_gb300 import fqt  # noqa: E402

EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 6


def _aligned(n=1 << 16):
    raw = ctypes.create_string_buffer(n + 256)
    return raw, ctypes.c_void_p((ctypes.addressof(raw) + 255) & ~255)


def _at(p, off):
    return ctypes.c_void_p(p.value + off)


def test_layer_norm_refusals():
    lib = fqt.load()
    raw, p = _aligned()

    def fwd(X=p, ldx=64, dtype=0, rows=4, cols=64, eps=1e-5, Y=p, ldy=64, mean=p):
        return lib.fqt_layer_norm_forward(X, ldx, dtype, rows, cols, p, p, eps, Y, ldy, mean, p,
                                          None)

    assert fwd(X=None) == EINVAL and fwd(Y=None) == EINVAL
    assert fwd(dtype=2) == EINVAL
    assert fwd(rows=-1) == EINVAL and fwd(cols=0) == EINVAL and fwd(cols=(1 << 30) + 1) == EINVAL
    assert fwd(ldx=63) == EINVAL and fwd(ldy=63) == EINVAL and fwd(ldx=1 << 62) == EINVAL
    assert fwd(X=_at(p, 2)) == EINVAL and fwd(Y=_at(p, 1), dtype=1) == EINVAL
    assert fwd(mean=_at(p, 2)) == EINVAL
    for eps in (-1e-5, float("nan"), float("inf")):
        assert fwd(eps=eps) == EINVAL
    assert fwd(rows=0, X=None, Y=None) == 0

    def bwd(dY=p, lddy=64, X=p, mean=p, dX=p, dg=p, db=p, ws=p, nbytes=1 << 30, rows=4, cols=64):
        return lib.fqt_layer_norm_backward(dY, lddy, X, 64, 0, rows, cols, mean, p, p, dX, 64, dg,
                                           db, ws, nbytes, None)

    assert bwd(dY=None) == EINVAL and bwd(X=None) == EINVAL and bwd(mean=None) == EINVAL
    assert bwd(lddy=10) == EINVAL and bwd(cols=0) == EINVAL and bwd(rows=-1) == EINVAL
    assert bwd(dX=None, dg=None, db=None) == EINVAL
    assert bwd(dg=_at(p, 2)) == EINVAL
    assert bwd(ws=None) == EWORKSPACE and bwd(nbytes=256) == EWORKSPACE
    assert bwd(ws=_at(p, 16)) == EWORKSPACE
    del raw
