"""Code matrices whose rows are too far apart for 64-bit offsets, or for the tensor maps
of a product, are refused before any CUDA call (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2010_14298_gb300 import fqt

EINVAL = 1


@pytest.mark.parametrize("pitch", [1 << 40, 1 << 41, 1 << 60])
def test_pitches_past_the_limit(pitch):
    lib = fqt.load()
    raw = torch.zeros((1 << 16) + 256, dtype=torch.uint8)
    at = (raw.data_ptr() + 255) & ~255
    p = ctypes.c_void_p(at)

    def f8(rows, pitch):
        return fqt._F8(rows, 64, pitch, 1, 0, at, at)

    far, near, none = f8(4, pitch), f8(4, 64), None
    for q, qt in ((far, none), (none, far), (near, far)):
        assert lib.fqt_quantize_fp8(p, 64, 0, 4, 64, 1, q and ctypes.byref(q),
                                    qt and ctypes.byref(qt), p, 256, None) == EINVAL
    for a, b in ((far, near), (near, far)):
        assert lib.fqt_fp8_matmul(ctypes.byref(a), ctypes.byref(b), 0, p, 4, p, 256,
                                  None) == EINVAL
