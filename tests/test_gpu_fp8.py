"""Products of 8-bit floating-point codes with a scale per block of 128, and their
quantizer, against plain implementations in 64 bits.

Tolerances.  The quantizer is exact: scales and codes are compared bit for bit.  In a
product the terms are exact; each step of 32 of them rounds its sum to the fp32
accumulator, at worst by truncation, which drops under 2^-23 of the running magnitude
(at most S, the sum of all magnitudes), and accumulators of several parts add as many
roundings as there are parts: |error| <= (K / 32 + 20) 2^-23 S.  A bf16 output adds
2^-8 of itself.
"""
import numpy as np
import pytest
import torch

from paper_2010_14298_gb300 import fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _matrix(rows, cols, dtype, seed, gap=0, scale=1.0):
    g = _gen(seed)
    x = torch.randn(rows, cols + gap, generator=g, device="cuda")
    x *= torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda")) * scale
    return x.to(DTYPES[dtype])[:, gap // 2:gap // 2 + cols]


# --- the quantizer, in numpy ------------------------------------------------
E4M3 = np.array([(-1.0) ** (c >> 7) * ((c & 7) * 2.0 ** -9 if (c >> 3 & 15) == 0 else
                                        (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                 if c & 127 != 127 else np.nan for c in range(256)])


def _codes(v):
    """The codes of |v| <= 448: by distance to all values, ties to the even code."""
    pos = E4M3[:127]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (c + 128 * np.signbit(v)).astype(np.uint8)


def _exponent(amax):
    m, e = np.frexp(amax)
    e = np.where(m > 0.875, e - 8, e - 9)
    return np.where(amax > 0, np.clip(e, -127, 127), 0)


def _reference(x, block_rows):
    """(codes, scales by block) of a finite matrix, its blocks along the rows."""
    rows, cols = x.shape
    nb = -(-cols // 128)
    codes = np.zeros((rows, cols), np.uint8)
    scales = np.zeros((nb, rows))
    for k in range(nb):
        part = x[:, 128 * k:128 * (k + 1)]
        amax = np.abs(part).max(1)
        if block_rows == 128:
            for r in range(0, rows, 128):
                amax[r:r + 128] = amax[r:r + 128].max()
        e = _exponent(amax)
        scales[k] = np.ldexp(1.0, e)
        codes[:, 128 * k:128 * (k + 1)] = _codes(part / scales[k][:, None])
    return codes, scales


def _scales(q):
    """By block and row."""
    e = q.scales.cpu().numpy()[:, :q.rows].astype(int) - 127
    return np.ldexp(1.0, e.transpose(0, 2, 1).reshape(-1, q.rows)[:-(-q.cols // 128)])


def _check_codes(q, x, block_rows):
    codes, scales = _reference(x, block_rows)
    got = q.codes.cpu().numpy()[:, :q.cols]
    assert np.array_equal(_scales(q), scales)
    assert np.array_equal(got, codes)


def test_reference_codes_are_e4m3():
    """The table and the rounding of this file against PyTorch's conversion."""
    c = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(c).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(t, nan=-1.0), np.nan_to_num(E4M3, nan=-1.0))
    v = np.random.default_rng(0).uniform(-448, 448, 20000).astype(np.float32)
    v = np.concatenate([v, v * 2.0 ** -14, E4M3[:126] + np.diff(E4M3[:127]) / 2, [0.0, -0.0]])
    v = v.astype(np.float32)
    t = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(t, _codes(v.astype(np.float64)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,gap", [(1, 1, 0), (1, 1024, 0), (5, 128, 8), (127, 129, 3),
                                           (128, 128, 0), (300, 515, 0), (1000, 336, 16),
                                           (129, 1201, 402), (640, 40, 0)])
def test_quantizer_is_exact(rows, cols, gap, block_rows, dtype):
    X = _matrix(rows, cols, dtype, rows + cols, gap)
    x = X.double().cpu().numpy()
    ws = fqt.Workspace.of_size(256)
    q, qt = fqt.quantize_fp8(X, block_rows, cols=True, ws=ws)
    assert fqt.sync_status(ws) == 0
    assert q.shape == (rows, cols) and qt.shape == (cols, rows)
    assert q.block_rows == qt.block_rows == block_rows
    _check_codes(q, x, block_rows)
    _check_codes(qt, np.ascontiguousarray(x.T), block_rows)
    only, none = fqt.quantize_fp8(X, block_rows)
    assert none is None and torch.equal(only.codes[:, :cols], q.codes[:, :cols])
    none, only = fqt.quantize_fp8(X, block_rows, rows=False, cols=True)
    assert none is None and torch.equal(only.codes[:, :rows], qt.codes[:, :rows])
    want = torch.from_numpy(E4M3)[q.codes[:, :cols].cpu().long()] \
        * torch.from_numpy(_scales(q).T).repeat_interleave(128, 1)[:, :cols]
    assert torch.equal(q.dequantize().double().cpu(), want)


def test_blocks_at_the_ends_of_the_range():
    """Zeros, subnormal entries, the largest finite ones, and maxima on and next to
    448 times a power of two."""
    x = np.zeros((16, 256), np.float32)
    x[1, :3] = [1e-44, -3e-42, 1e-45]
    x[2, :2] = [3.4028235e38, -1.0]
    x[3, 130] = 448.0
    x[4, 0] = np.nextafter(np.float32(448.0), np.float32(1e9))
    x[5, 0] = np.nextafter(np.float32(448.0), np.float32(0))
    x[6, :2] = [448.0 * 2.0 ** -100, 2.0 ** -109]
    x[7] = -0.0
    x[8, :2] = [1.1754944e-38, 1e-39]
    q, qt = fqt.quantize_fp8(torch.from_numpy(x).cuda(), cols=True)
    _check_codes(q, x.astype(np.float64), 1)
    _check_codes(qt, np.ascontiguousarray(x.T).astype(np.float64), 1)


def test_bf16_blocks_at_the_ends_of_the_range():
    """Subnormal, smallest and largest bf16 entries, alone and beside larger ones."""
    bits = torch.zeros((16, 256), dtype=torch.int16)
    bits[1, :4] = torch.tensor([1, 3, 0x7F, -32768 + 5], dtype=torch.int16)
    bits[2, :2] = torch.tensor([0x7F7F, 1], dtype=torch.int16)
    bits[3, :3] = torch.tensor([0x80, 0x40, 0x81], dtype=torch.int16)
    bits[4, 128:131] = torch.tensor([0x3F80, 0x0100, 0x3B00], dtype=torch.int16)
    bits[5, :3] = torch.tensor([0x43E0, 0x43E1, 0x43DF], dtype=torch.int16)
    X = bits.view(torch.bfloat16)
    q, qt = fqt.quantize_fp8(X.cuda(), cols=True)
    only, _ = fqt.quantize_fp8(X.cuda())
    x = X.double().numpy()
    _check_codes(q, x, 1)
    _check_codes(only, x, 1)
    _check_codes(qt, np.ascontiguousarray(x.T), 1)


def test_entries_that_are_not_finite():
    """They take the NaN code, count for no scale, and are reported."""
    X = _matrix(200, 300, "bf16", 1)
    bad = X.clone()
    bad[3, 5], bad[150, 299], bad[150, 0] = float("inf"), float("nan"), float("-inf")
    ws = fqt.Workspace.of_size(256)
    q, qt = fqt.quantize_fp8(bad, cols=True, ws=ws)
    assert fqt.sync_status(ws) == 4 and fqt.sync_status(ws) == 0
    X[3, 5] = X[150, 299] = X[150, 0] = 0
    codes, scales = _reference(X.double().cpu().numpy(), 1)
    got = q.codes.cpu().numpy()[:, :300]
    at = [(3, 5), (150, 299), (150, 0)]
    only, _ = fqt.quantize_fp8(bad)
    assert torch.equal(only.codes[:, :300], q.codes[:, :300])
    tcodes, tscales = _reference(np.ascontiguousarray(X.double().cpu().numpy().T), 1)
    assert np.array_equal(_scales(qt), tscales)
    for r, c in at:
        assert got[r, c] & 127 == 127 and qt.codes[c, r].item() & 127 == 127
        got[r, c] = codes[r, c]
    assert np.array_equal(got, codes)
    assert np.array_equal(_scales(q), scales)
    # a product shows it in its rows alone
    out = fqt.fp8_matmul(q, fqt.quantize_fp8(torch.ones((4, 300), device="cuda"))[0])
    nan = torch.isnan(out).any(1).nonzero().flatten().tolist()
    assert nan == [3, 150]


def _product_bound(A, B):
    return (A.shape[1] / 32 + 20) * 2.0 ** -23 * (A.abs() @ B.abs().t())


def _values64(q):
    return q.dequantize().double()


SIZES = [(1, 16, 1), (1, 4096, 1024), (3, 300, 129), (33, 1000, 200), (64, 4096, 1024),
         (65, 64, 128), (128, 128, 128), (129, 257, 385), (200, 1201, 1523), (336, 1201, 1523),
         (1523, 336, 1201), (2048, 2304, 512), (4096, 2560, 384), (5000, 4097, 40),
         (17, 50000, 100), (40000, 24, 300), (100, 90, 8200), (300, 200, 70000), (2304, 2100, 9000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product_matches_64_bits(M, N, K, dtype):
    a, _ = fqt.quantize_fp8(_matrix(M, K, "f32", 1))
    for block_rows in (1, 128):
        b, _ = fqt.quantize_fp8(_matrix(N, K, "f32", 2), block_rows)
        ws = fqt.Workspace.of_size(fqt.fp8_matmul_workspace_size(M, N, K))
        out = fqt.fp8_matmul(a, b, dtype=DTYPES[dtype], ws=ws)
        assert fqt.sync_status(ws) == 0
        A, B = _values64(a), _values64(b)
        want = A @ B.t()
        bound = _product_bound(A, B)
        if dtype == "bf16":
            bound = bound + 2.0 ** -8 * want.abs()
        assert out.dtype == DTYPES[dtype] and out.shape == (M, N)
        assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1024, 4096), (2, 131, 1700), (33, 300, 5000), (64, 257, 8192),
                                   (65, 66, 1665), (100, 333, 2900), (130, 1900, 2048),
                                   (257, 129, 20000)])
def test_tiles_whose_blocks_are_shared(M, N, K, dtype):
    """Few tiles and a long contraction: CTAs share the K blocks of a tile; the output in
    wider rows, of which nothing else is written, and the same bits again."""
    a, _ = fqt.quantize_fp8(_matrix(M, K, "bf16", 1))
    b, _ = fqt.quantize_fp8(_matrix(N, K, "bf16", 2), 128)
    A, B = _values64(a), _values64(b)
    want, bound = A @ B.t(), _product_bound(A, B)
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * want.abs()
    wide = torch.full((M + 1, N + 5), 7.0, dtype=DTYPES[dtype], device="cuda")
    ws = fqt.Workspace.of_size(fqt.fp8_matmul_workspace_size(M, N, K))
    fqt.fp8_matmul(a, b, out=wide[:M, :N], ws=ws)
    assert fqt.sync_status(ws) == 0
    assert ((wide[:M, :N].double() - want).abs() <= bound).all()
    assert (wide[M:] == 7).all() and (wide[:, N:] == 7).all()
    assert torch.equal(fqt.fp8_matmul(a, b, dtype=DTYPES[dtype], ws=ws), wide[:M, :N])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(207, 59, 27), (195, 21, 1064), (81, 7, 121), (300, 1201, 330),
                                   (767, 885, 129), (3000, 2045, 200), (5, 131, 300),
                                   (100, 90, 8200)])
def test_nothing_past_the_rows_is_read_or_written(M, N, K, dtype):
    """Outputs of 1 to 8 entries in wider rows, whatever alignment that gives them, and
    codes between whose rows lie other bytes."""
    a, _ = fqt.quantize_fp8(_matrix(M, K, "f32", 1))
    b, _ = fqt.quantize_fp8(_matrix(N, K, "f32", 2))
    A, B = _values64(a), _values64(b)
    want, bound = A @ B.t(), _product_bound(A, B)
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * want.abs()
    for q in (a, b):
        q.codes[:, K:] = 0x7F  # not a number
    for gap in range(1, 9):
        wide = torch.full((M + 1, N + gap), 7.0, dtype=DTYPES[dtype], device="cuda")
        fqt.fp8_matmul(a, b, out=wide[:M, :N])
        assert ((wide[:M, :N].double() - want).abs() <= bound).all(), gap
        assert (wide[M:] == 7).all() and (wide[:, N:] == 7).all(), gap


def test_scales_of_any_exponent():
    """Exponents from -127 on, with products of them inside fp32's range."""
    M, N, K = 150, 140, 1100
    a, _ = fqt.quantize_fp8(_matrix(M, K, "f32", 1))
    b, _ = fqt.quantize_fp8(_matrix(N, K, "f32", 2))
    for q, lo, hi in ((a, 0, 170), (b, 100, 180)):
        q.scales.copy_(torch.randint(lo, hi, q.scales.shape, generator=_gen(3), device="cuda"))
    A, B = _values64(a), _values64(b)
    out = fqt.fp8_matmul(a, b)
    # what lies under fp32's smallest normal number may be dropped
    assert ((out.double() - A @ B.t()).abs() <= _product_bound(A, B) + K * 2.0 ** -126).all()


def test_a_block_of_large_scale_does_not_hide_the_others():
    """One block's products cancel exactly; the small ones remain."""
    M, N, K = 130, 30, 384
    X = torch.zeros((M, K), device="cuda")
    W = torch.ones((N, K), device="cuda")
    X[:, 0], X[:, 1] = 2.0 ** 30, -2.0 ** 30
    X[:, 200] = 1.0
    out = fqt.fp8_matmul(fqt.quantize_fp8(X)[0], fqt.quantize_fp8(W)[0])
    assert (out == 1.0).all()


def test_layer_passes_and_their_shapes():
    """H = X~ W~^T, grad_X = dH~ W~, grad_W = dH~^T X~ from both orders of the codes."""
    T, C, D = 300, 200, 150
    X, W, dH = (_matrix(r, c, "bf16", s) for r, c, s in ((T, D, 1), (C, D, 2), (T, C, 3)))
    qx, qxt = fqt.quantize_fp8(X, cols=True)
    qw, qwt = fqt.quantize_fp8(W, 128, cols=True)
    qd, qdt = fqt.quantize_fp8(dH, cols=True)
    assert torch.equal(qw.dequantize(), qwt.dequantize().t())
    for got, l, r in ((fqt.fp8_matmul(qx, qw), qx, qw), (fqt.fp8_matmul(qd, qwt), qd, qwt),
                      (fqt.fp8_matmul(qdt, qxt), qdt, qxt)):
        A, B = _values64(l), _values64(r)
        assert ((got.double() - A @ B.t()).abs() <= _product_bound(A, B)).all()


def test_output_rows_and_repeated_calls():
    """An output inside wider rows, bits that do not change, a shared workspace."""
    M, N, K = 700, 129, 2000
    a, b = fqt.quantize_fp8(_matrix(M, K, "f32", 1))[0], fqt.quantize_fp8(_matrix(N, K, "f32", 2))[0]
    ws = fqt.Workspace.of_size(fqt.fp8_matmul_workspace_size(M, N, K))
    ref = fqt.fp8_matmul(a, b, ws=ws)
    wide = torch.full((M, 200), 5.0, device="cuda")
    fqt.fp8_matmul(a, b, out=wide[:, 30:159], ws=ws)
    assert torch.equal(wide[:, 30:159], ref)
    assert (wide[:, :30] == 5).all() and (wide[:, 159:] == 5).all()
    for _ in range(3):
        assert torch.equal(fqt.fp8_matmul(a, b, ws=ws), ref)


def test_empty_sizes():
    a = fqt.quantize_fp8(torch.empty((0, 64), device="cuda"))[0]
    b = fqt.quantize_fp8(torch.ones((8, 64), device="cuda"))[0]
    assert fqt.fp8_matmul(a, b).shape == (0, 8)
    assert fqt.fp8_matmul(b, a).shape == (8, 0)
    _, t = fqt.quantize_fp8(torch.empty((0, 64), device="cuda"), cols=True)
    out = torch.full((64, 64), 3.0, device="cuda")
    assert (fqt.fp8_matmul(t, t, out=out) == 0).all()


def test_another_stream_and_graphs():
    X, W = _matrix(500, 700, "bf16", 1), _matrix(600, 700, "bf16", 2)
    qw = fqt.quantize_fp8(W, 128)[0]
    ref = fqt.fp8_matmul(fqt.quantize_fp8(X)[0], qw)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = fqt.fp8_matmul(fqt.quantize_fp8(X, stream=s)[0], qw, stream=s)
    s.synchronize()
    assert torch.equal(out, ref)
    q, o = fqt.Fp8Tensor.empty(500, 700), torch.zeros_like(ref)
    ws = fqt.Workspace.of_size(fqt.fp8_matmul_workspace_size(500, 600, 700))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fqt.quantize_fp8(X, q=q, ws=ws)
        fqt.fp8_matmul(q, qw, out=o, ws=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, ref)


def test_refusals():
    X = torch.zeros((4, 64), device="cuda")
    q, _ = fqt.quantize_fp8(X)
    for bad in (lambda: fqt.quantize_fp8(X.cpu()), lambda: fqt.quantize_fp8(X[0]),
                lambda: fqt.quantize_fp8(X, q=fqt.Fp8Tensor.empty(64, 4)),
                lambda: fqt.quantize_fp8(X, qt=fqt.Fp8Tensor.empty(4, 64)),
                lambda: fqt.quantize_fp8(X, q=fqt.Fp8Tensor.empty(4, 64, device="cpu")),
                lambda: fqt.fp8_matmul(q, fqt.Fp8Tensor.empty(4, 65)),
                lambda: fqt.fp8_matmul(q, q, out=torch.zeros((4, 5), device="cuda")),
                lambda: fqt.fp8_matmul(q, q, out=torch.zeros((4, 4))),
                lambda: fqt.fp8_matmul(q, fqt.Fp8Tensor.empty(4, 64, device="cpu"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        fqt.quantize_fp8(X.half())
    with pytest.raises(TypeError):
        fqt.fp8_matmul(q, q, dtype=torch.float16)
    with pytest.raises((fqt.FqtError, ValueError)):
        fqt.quantize_fp8(X, block_rows=64)
    with pytest.raises(fqt.FqtError) as e:
        fqt.fp8_matmul(q, q, ws=fqt.Workspace.of_size(128))
    assert e.value.status == 6
