"""Layer norm, forward and backward, against its formula in 64 bits.

Tolerances.  With u = 2^-24, a row's sums of n terms accumulate in short chains
(at most 32 terms a thread in the kernels that hold a row, n / 1024 in those that do
not, then trees), so a sum is off by at most 64 u times the sum of the magnitudes
here.  y and dx are formed from those by under ten roundings of terms no larger than
a few times the row's largest entry of (x - mean) rstd gamma (or of the gradient's
terms), hence 1e-5 of that; bf16 outputs add half a unit in the eighth bit, 2^-8.  The
column sums add up to rows / CTAs terms in a chain: 1e-5 of the sum of magnitudes.
"""
import numpy as np
import pytest
import torch

from paper_2010_14298_gb300 import fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}
EPS = 1e-5


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _matrix(rows, cols, dtype, gap, seed, scale=1.0, offset=0.0):
    """rows x cols inside rows of cols + gap entries, one entry in."""
    g = _gen(seed)
    wide = torch.randn(rows, cols + gap, generator=g, device="cuda") * scale + offset
    wide = wide.to(DTYPES[dtype])
    return wide[:, gap // 2:gap // 2 + cols]


def _fwd64(X, gamma, beta):
    x = X.double()
    mean = x.mean(1, keepdim=True)
    rstd = (((x - mean) ** 2).mean(1, keepdim=True) + EPS) ** -0.5
    y = (x - mean) * rstd
    if gamma is not None:
        y = y * gamma.double()
    if beta is not None:
        y = y + beta.double()
    return y, mean[:, 0], rstd[:, 0]


def _bwd64(dY, X, mean, rstd, gamma):
    dy, x = dY.double(), X.double()
    xh = (x - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy if gamma is None else dy * gamma.double()
    dx = rstd.double()[:, None] * (g - g.mean(1, keepdim=True)
                                   - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), (dy * xh).abs().sum(0), dy.abs().sum(0)


# one token, one column, rows of every kernel's kind: 16-byte entries, single entries
# (odd lengths, odd pitches), one and two per thread, wider than a CTA's registers;
# rows fewer than the SMs, and enough for two at a time
SHAPES = [(1, 1, 0), (1, 1024, 0), (3, 2, 0), (7, 8, 0), (5, 31, 2), (64, 33, 0), (300, 335, 0),
          (1523, 1201, 402), (100, 1000, 8), (200, 1000, 3), (5000, 64, 0), (9000, 256, 16),
          (3000, 4096, 0), (40, 4100, 4), (33, 8200, 0), (20, 16384, 0), (9, 8191, 0),
          (6, 20011, 0), (3, 40000, 0), (700, 33000, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,gap", SHAPES)
def test_forward_matches_the_formula(rows, cols, gap, dtype):
    X = _matrix(rows, cols, dtype, gap, rows + cols, 2.0, 0.7)
    g = _gen(3)
    gamma = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    beta = 0.1 * torch.randn(cols, generator=g, device="cuda")
    for ga, be in ((gamma, beta), (None, None)):
        Y, mean, rstd = fqt.layer_norm_forward(X, ga, be, EPS)
        y, m, r = _fwd64(X, ga, be)
        amax = X.double().abs().amax(1)
        assert ((mean.double() - m).abs() <= 64 * 2.0 ** -24 * amax).all()
        # the variance is off by 64 u of itself and the square of the mean's error
        assert ((rstd.double() - r).abs() <= 1e-5 * r).all()
        assert Y.dtype == X.dtype and Y.shape == X.shape
        top = y.abs().amax(1, keepdim=True)
        assert ((Y.double() - y).abs() <= (1e-5 * top + ROUND[dtype] * y.abs() + 1e-5)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,gap", SHAPES)
def test_backward_matches_the_formula(rows, cols, gap, dtype):
    X = _matrix(rows, cols, dtype, gap, rows + cols, 2.0, 0.7)
    dY = _matrix(rows, cols, dtype, gap // 2, rows + cols + 1)
    gamma = 1 + 0.2 * torch.randn(cols, generator=_gen(4), device="cuda")
    _, mean, rstd = fqt.layer_norm_forward(X, gamma, None, EPS)
    for ga in (gamma, None):
        dX, dgamma, dbeta = fqt.layer_norm_backward(dY, X, mean, rstd, ga)
        dx, dg, db, dg_abs, db_abs = _bwd64(dY, X, mean, rstd, ga)
        # the three terms that dx is the difference of
        top = rstd.double()[:, None] * (dY.double().abs() * (1.0 if ga is None else
                                                             ga.double().abs())
                                        ).amax(1, keepdim=True) * max(1.0, cols ** 0.5)
        assert ((dX.double() - dx).abs() <= 1e-5 * top + ROUND[dtype] * dx.abs()).all()
        assert ((dgamma.double() - dg).abs() <= 1e-5 * dg_abs).all()
        assert ((dbeta.double() - db).abs() <= 1e-5 * db_abs).all()


def test_a_mean_far_from_zero_keeps_its_variance():
    """Deviations of 1 about 4096: a sum of squares in 32 bits would lose them (its
    24 bits end at 1 where the squares are 2^24)."""
    X = _matrix(50, 1000, "f32", 0, 9, 1.0, 4096.0)
    Y, mean, rstd = fqt.layer_norm_forward(X, None, None, EPS)
    y, m, r = _fwd64(X, None, None)
    # the mean is off by up to 2^-11, which moves every entry by that
    assert ((Y.double() - y).abs() <= 1e-3).all()
    assert ((rstd.double() - r).abs() <= 1e-5 * r).all()


def test_gradients_match_differences():
    """dX against central differences of the loss sum(dY * Y) in 64 bits, with the
    kernel's own statistics; h = 1e-4 leaves h^2 and 1e-16 / h behind."""
    rows, cols = 3, 37
    X = _matrix(rows, cols, "f32", 0, 21)
    dY = _matrix(rows, cols, "f32", 0, 22)
    gamma = 1 + 0.2 * torch.randn(cols, generator=_gen(23), device="cuda")
    beta = torch.zeros(cols, device="cuda")
    _, mean, rstd = fqt.layer_norm_forward(X, gamma, beta, EPS)
    dX, dgamma, dbeta = fqt.layer_norm_backward(dY, X, mean, rstd, gamma)
    x, ga, be, d = (t.double().cpu() for t in (X, gamma, beta, dY))

    def loss(x, ga, be):
        return (_fwd64(x, ga, be)[0] * d).sum()

    h = 1e-4
    for got, at in ((dX, 0), (dgamma, 1), (dbeta, 2)):
        args = [x, ga, be]
        got = got.double().cpu().reshape(-1)
        for i in range(0, got.numel(), 5):
            up, down = args[at].clone(), args[at].clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            args_up, args_down = list(args), list(args)
            args_up[at], args_down[at] = up, down
            diff = (loss(*args_up) - loss(*args_down)) / (2 * h)
            assert abs(float(diff - got[i])) <= 1e-4 * (1 + abs(float(diff)))


def test_a_row_that_is_not_finite_stays_alone():
    X = _matrix(40, 1024, "bf16", 0, 5)
    clean, _, _ = fqt.layer_norm_forward(X)
    X = X.clone()
    X[7, 100], X[11, 3] = float("inf"), float("nan")
    Y, mean, rstd = fqt.layer_norm_forward(X)
    for r in (7, 11):
        assert torch.isnan(Y[r]).all()
    keep = [r for r in range(40) if r not in (7, 11)]
    assert torch.equal(Y[keep], clean[keep])


def test_constant_rows():
    """No variance: y = beta, rstd = eps^(-1/2)."""
    X = torch.full((5, 300), 3.0, device="cuda")
    beta = torch.randn(300, generator=_gen(1), device="cuda")
    Y, mean, rstd = fqt.layer_norm_forward(X, None, beta, 1e-5)
    assert torch.equal(Y, beta.expand(5, 300))
    assert ((rstd.double() - 1e-5 ** -0.5).abs() <= 1e-4).all()


def test_no_rows():
    X = torch.empty((0, 64), device="cuda")
    Y, mean, rstd = fqt.layer_norm_forward(X)
    assert Y.shape == (0, 64)
    dg = torch.full((64,), 7.0, device="cuda")
    dX, dgamma, dbeta = fqt.layer_norm_backward(X, X, mean, rstd, out_gamma=dg)
    assert dX.shape == (0, 64) and (dgamma == 0).all() and (dbeta == 0).all()


def test_one_direction_alone_and_the_same_bits_again():
    X, dY = _matrix(999, 768, "bf16", 0, 1), _matrix(999, 768, "bf16", 0, 2)
    _, mean, rstd = fqt.layer_norm_forward(X)
    dX, dgamma, dbeta = fqt.layer_norm_backward(dY, X, mean, rstd)
    only_x = fqt.layer_norm_backward(dY, X, mean, rstd, grad_w=False)
    only_w = fqt.layer_norm_backward(dY, X, mean, rstd, grad_x=False)
    assert only_x[1] is None and only_x[2] is None and only_w[0] is None
    assert torch.equal(only_x[0], dX)
    assert torch.equal(only_w[1], dgamma) and torch.equal(only_w[2], dbeta)


def test_outputs_in_wider_rows_and_other_layouts():
    """Outputs keep to their columns; transposed and broadcast inputs are read.
    (Rows that are not on 16 bytes are summed in another order.)"""
    X = _matrix(70, 96, "f32", 0, 8)
    wide = torch.full((70, 130), 5.0, device="cuda")
    Y, _, _ = fqt.layer_norm_forward(X, out=wide[:, 20:116])
    ref, mean, rstd = fqt.layer_norm_forward(X)
    y = _fwd64(X, None, None)[0]
    top = y.abs().amax(1, keepdim=True)
    for got in (wide[:, 20:116], ref):
        assert ((got.double() - y).abs() <= 1e-5 * top).all()
    assert (wide[:, :20] == 5).all() and (wide[:, 116:] == 5).all()
    t, _, _ = fqt.layer_norm_forward(X.t().contiguous().t())
    assert torch.equal(t, ref)
    b, _, _ = fqt.layer_norm_forward(X[:1].expand(4, 96))
    assert torch.equal(b, ref[:1].expand(4, 96))


def test_another_stream():
    X = _matrix(4000, 1024, "bf16", 0, 8)
    dY = _matrix(4000, 1024, "bf16", 0, 9)
    ref, mean, rstd = fqt.layer_norm_forward(X)
    want = fqt.layer_norm_backward(dY, X, mean, rstd)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    Y, m, r = fqt.layer_norm_forward(X, stream=s)
    got = fqt.layer_norm_backward(dY, X, m, r, stream=s)
    s.synchronize()
    assert torch.equal(Y, ref) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_graph_capture():
    X = _matrix(500, 1024, "bf16", 0, 8)
    ws = fqt.Workspace.of_size(fqt.layer_norm_workspace_size(500, 1024))
    Y, mean, rstd = fqt.layer_norm_forward(X)
    dX, dg, db = fqt.layer_norm_backward(X, X, mean, rstd, ws=ws)
    want = [t.clone() for t in (Y, dX, dg, db)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fqt.layer_norm_forward(X, out=Y, mean=mean, rstd=rstd)
        fqt.layer_norm_backward(X, X, mean, rstd, ws=ws, out_x=dX, out_gamma=dg, out_beta=db)
    for t in (Y, dX, dg, db):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((Y, dX, dg, db), want))


def test_refusals():
    X = torch.zeros((4, 64), device="cuda")
    v = torch.zeros(64, device="cuda")
    m = torch.ones(4, device="cuda")
    for bad in (lambda: fqt.layer_norm_forward(X.cpu()),
                lambda: fqt.layer_norm_forward(X[0]),
                lambda: fqt.layer_norm_forward(X, v[:32]),
                lambda: fqt.layer_norm_forward(X, v.bfloat16()),
                lambda: fqt.layer_norm_forward(X, out=torch.zeros((4, 32), device="cuda")),
                lambda: fqt.layer_norm_forward(X, out=X.bfloat16()),
                lambda: fqt.layer_norm_forward(X, out=torch.zeros((64, 4), device="cuda").t()),
                lambda: fqt.layer_norm_backward(X[:2], X, m, m),
                lambda: fqt.layer_norm_backward(X, X, m[:2], m),
                lambda: fqt.layer_norm_backward(X.bfloat16(), X, m, m)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        fqt.layer_norm_forward(X.half())
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(fqt.FqtError) as e:
            fqt.layer_norm_forward(X, eps=eps)
        assert e.value.status == 1
    small = fqt.Workspace.of_size(512)
    with pytest.raises(fqt.FqtError) as e:
        fqt.layer_norm_backward(X, X, m, m, ws=small)
    assert e.value.status == 6


@pytest.mark.parametrize("cols", [1, 3, 7, 24, 48, 335, 768, 1000, 1201, 4096, 8190, 8192])
def test_means_are_rounded_quotients(cols):
    """Sums of small integers are exact in any order, so the mean that is nearest to the
    quotient is the only one; rows of equal entries have no variance."""
    rows = 400
    X = torch.randint(-1000, 1001, (rows, cols), generator=_gen(cols), device="cuda").float()
    X[0], X[1] = 1000.0, -999.0
    X[2] = torch.randint(1, 1001, (cols,), generator=_gen(cols + 1), device="cuda").float()
    Y, mean, rstd = fqt.layer_norm_forward(X, eps=EPS)
    want = (X.double().sum(1) / cols).float()
    assert torch.equal(mean, want)
    assert (Y[:2] == 0).all()
    assert ((rstd[:2].double() - EPS ** -0.5).abs() <= 8 * 2.0 ** -24 * EPS ** -0.5).all()


# 32 entries a thread: with and without rows fetched ahead, with a last row that is not
# full, past what 16 entries hold; and the widths beside which it goes back to 16
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,gap", [(1000, 1024, 0), (2600, 1000, 8), (300, 8192, 0),
                                           (700, 8000, 0), (160, 16384, 0), (310, 16376, 8),
                                           (153, 10000, 0), (400, 5120, 16), (3000, 1088, 0),
                                           (500, 640, 0), (700, 6144, 0), (5000, 520, 8)])
def test_forward_of_wide_groups(rows, cols, gap, dtype):
    test_forward_matches_the_formula(rows, cols, gap, dtype)
