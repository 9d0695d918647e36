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


def test_fp8_refusals():
    lib = fqt.load()
    raw, p = _aligned()

    def f8(rows, cols, pitch=None, block_rows=1, codes=p.value, scales=p.value):
        return fqt._F8(rows, cols, -(-cols // 16) * 16 if pitch is None else pitch, block_rows, 0,
                       codes, scales)

    def quant(q, qt=None, X=p, ldx=64, dtype=0, rows=4, cols=64, br=1, ws=p, nbytes=256):
        return lib.fqt_quantize_fp8(X, ldx, dtype, rows, cols, br,
                                    ctypes.byref(q) if q else None,
                                    ctypes.byref(qt) if qt else None, ws, nbytes, None)

    good = f8(0, 0, 64)
    assert quant(None) == EINVAL
    assert quant(good, X=None) == EINVAL and quant(good, X=_at(p, 2)) == EINVAL
    assert quant(good, br=64) == EINVAL and quant(good, dtype=3) == EINVAL
    assert quant(good, rows=-1) == EINVAL and quant(good, cols=0) == EINVAL
    assert quant(good, rows=(1 << 22) + 1) == EINVAL and quant(good, ldx=60) == EINVAL
    assert quant(f8(0, 0, 48)) == EINVAL              # rows of 64 codes in 48 bytes
    assert quant(f8(0, 0, 72)) == EINVAL              # no multiple of 16
    assert quant(f8(0, 0, 64, codes=p.value + 8)) == EINVAL
    assert quant(f8(0, 0, 64, scales=None)) == EINVAL
    assert quant(good, qt=f8(0, 0, 0)) == EINVAL      # 4 codes in no bytes
    assert quant(good, ws=None) == EWORKSPACE and quant(good, nbytes=128) == EWORKSPACE
    assert quant(good, ws=_at(p, 8)) == EWORKSPACE
    assert quant(good, rows=0, X=None) == 0 and (good.rows, good.cols) == (0, 64)

    def mm(A, B, dtype=0, out=p, ldo=None, ws=p, nbytes=1 << 30):
        return lib.fqt_fp8_matmul(ctypes.byref(A) if A else None, ctypes.byref(B) if B else None,
                                  dtype, out, B.rows if ldo is None and B else ldo or 0, ws,
                                  nbytes, None)

    A, B = f8(10, 64), f8(20, 64)
    assert mm(None, B) == EINVAL and mm(A, None) == EINVAL and mm(A, B, dtype=2) == EINVAL
    assert mm(A, f8(20, 65)) == EINVAL and mm(A, f8(-1, 64)) == EINVAL
    assert mm(A, f8(20, 64, block_rows=2)) == EINVAL
    assert mm(A, f8(20, 64, pitch=48)) == EINVAL and mm(A, f8(20, 64, codes=None)) == EINVAL
    assert mm(A, B, out=None) == EINVAL and mm(A, B, out=_at(p, 2)) == EINVAL
    assert mm(A, B, ldo=19) == EINVAL
    assert mm(f8((1 << 22) + 1, 64), B) == EINVAL
    assert mm(A, B, ws=None) == EWORKSPACE and mm(A, B, nbytes=16) == EWORKSPACE
    assert mm(f8(0, 64), B) == 0 and mm(A, f8(0, 64)) == 0
    del raw


def test_fp8_tensors_that_do_not_fit_are_refused():
    u8 = dict(dtype=torch.uint8)
    codes, scales = torch.zeros((4, 64), **u8), torch.zeros((1, 128, 4), **u8)
    fqt.Fp8Tensor(codes, scales, 4, 64)
    for bad in (dict(codes=codes.int()), dict(scales=scales.float()), dict(rows=5),
                dict(cols=65), dict(codes=torch.zeros((4, 60), dtype=torch.uint8)),
                dict(scales=torch.zeros((1, 64, 4), **u8)),
                dict(scales=torch.zeros((2, 128, 4), **u8)),
                dict(codes=torch.zeros((64, 4), dtype=torch.uint8).t()), dict(block_rows=2)):
        with pytest.raises(ValueError):
            fqt.Fp8Tensor(**{**dict(codes=codes, scales=scales, rows=4, cols=64), **bad})


def test_clip_refusals():
    lib = fqt.load()
    raw, p = _aligned()

    def lst(*entries):
        a = (fqt._Tensor * max(1, len(entries)))()
        for i, e in enumerate(entries):
            a[i] = fqt._Tensor(*e)
        return a

    def call(grads, out=None, n=1, max_norm=1.0, norm=p, ws=p, nbytes=1 << 30):
        return lib.fqt_clip_grad_norm(grads, out, n, max_norm, norm, ws, nbytes, None)

    good = lst((p.value, 8, 0, 0))
    assert call(None) == EINVAL and call(good, n=-1) == EINVAL
    assert call(good, norm=None) == EINVAL           # nothing asked for
    assert call(good, norm=_at(p, 2)) == EINVAL
    assert call(lst((p.value, 8, 2, 0))) == EINVAL
    assert call(lst((p.value, -1, 0, 0))) == EINVAL
    assert call(lst((p.value, 1 << 41, 0, 0))) == EINVAL
    assert call(lst((None, 8, 0, 0))) == EINVAL
    assert call(lst((p.value + 2, 8, 0, 0))) == EINVAL
    assert call(lst((p.value + 1, 8, 1, 0))) == EINVAL
    assert call(good, out=lst((p.value, 7, 0, 0))) == EINVAL
    assert call(good, out=lst((p.value, 8, 1, 0))) == EINVAL
    assert call(good, out=good, max_norm=-1.0) == EINVAL
    assert call(good, out=good, max_norm=float("nan")) == EINVAL
    assert call(good, ws=None) == EWORKSPACE and call(good, nbytes=256) == EWORKSPACE
    assert call(good, ws=_at(p, 8)) == EWORKSPACE
    del raw


@pytest.mark.parametrize("calls", ["extension", "ctypes"])
def test_both_marshallings_take_and_refuse_the_same(calls):
    """The extension module's calls and the same through ctypes: what the library refuses
    (or has nothing to do for) without a GPU."""
    n = fqt.native() if calls == "extension" else fqt._CtypesCalls(fqt.load())
    X, v = torch.zeros(4, 64), torch.zeros(64)
    ws = torch.zeros(512, dtype=torch.uint8)
    assert n.layer_norm_forward(X, 64, 0, 4, 64, v, None, -1.0, X, 64, None, v, 0) == EINVAL
    assert n.layer_norm_forward(X, 64, 0, 0, 64, None, None, 1e-5, X, 64, v, v, 0) == 0
    assert n.layer_norm_backward(X, 64, X, 64, 0, -4, 64, v, v, None, X, 64, None, None, None, 0,
                                 0) == EINVAL
    q = fqt.Fp8Tensor.empty(4, 64, device="cpu")
    assert n.quantize_fp8(X, 64, 0, 4, 64, 2, q, None, ws, 512, 0) == EINVAL
    assert n.quantize_fp8(X, 64, 0, 4, 64, 1, None, None, ws, 512, 0) == EINVAL
    assert n.fp8_matmul(q, fqt.Fp8Tensor.empty(3, 65, device="cpu"), 0, X, 64, ws, 512, 0) == EINVAL
    assert n.clip_grad_norm(0, None, 1, 1.0, None, ws, 512, 0) == EINVAL
    a = (fqt._Tensor * 1)(fqt._Tensor(0, 5, 0, 0))
    assert n.clip_grad_norm(ctypes.addressof(a), None, 1, 1.0, v, ws, 512, 0) == EINVAL
