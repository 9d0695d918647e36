"""Layer norm's backward where the two terms that dX is corrected by are of order one.

Tolerances.  With u = 2^-24, a row's sums are chains of at most 32 terms (cols / 512 in
rows wider than a CTA's registers) and trees of under 32 additions: off by at most
c u sum |.|, c = 64 or cols / 512 + 32, whichever is more.  An entry
    dx = rstd (g - sum(g) / n - xh sum(g xh) / n)
takes under eight roundings of terms no larger than its own three, and inherits the
sums' errors: |error| <= rstd (8 u (|g| + |m1| + |xh m2|) + c u (mean|g| + |xh| mean|g xh|)).
A bf16 output adds 2^-8 of itself.
"""
import pytest
import torch

from paper_2010_14298_gb300 import fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}
U = 2.0 ** -24


def _case(rows, cols, dtype, gap=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + cols)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X = (2 * randn(rows, cols + gap) + 0.7).to(DTYPES[dtype])[:, gap // 2:gap // 2 + cols]
    _, mean, rstd = fqt.layer_norm_forward(X)
    xh = (X.float() - mean[:, None]) * rstd[:, None]
    dY = (randn(rows, cols) + 0.5 + 0.7 * xh).to(DTYPES[dtype])
    return X, dY, mean, rstd, 1 + 0.2 * randn(cols)


def _check(dX, X, dY, mean, rstd, gamma, dtype):
    x, dy, r = X.double(), dY.double(), rstd.double()[:, None]
    xh = (x - mean.double()[:, None]) * r
    g = dy if gamma is None else dy * gamma.double()
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - m1 - xh * m2)
    c = max(64, X.shape[1] / 512 + 32)
    bound = r * (8 * U * (g.abs() + m1.abs() + (xh * m2).abs())
                 + c * U * (g.abs().mean(1, keepdim=True)
                            + xh.abs() * (g * xh).abs().mean(1, keepdim=True)))
    bound = bound + ROUND[dtype] * dx.abs()
    assert ((dX.double() - dx).abs() <= bound).all()
    # a lost or a misweighted term would show
    for wrong in (r * (g - xh * m2), r * (g - m1), r * (g - m1 - xh * m2 * (1 + 1 / 16)),
                  r * (g - m1 * (1 + 1 / 16) - xh * m2)):
        assert ((wrong - dx).abs() > bound).any(1).all()


SHAPES = [(300, 335, 0), (1523, 1201, 402), (100, 1000, 8), (200, 1000, 3), (9000, 256, 16),
          (3000, 4096, 0), (400, 8192, 0), (33, 8200, 0), (40, 8193, 0), (6, 20011, 0),
          (20, 16384, 0), (7, 40000, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,gap", SHAPES)
def test_the_terms_of_dx(rows, cols, gap, dtype):
    X, dY, mean, rstd, gamma = _case(rows, cols, dtype, gap)
    for ga in (gamma, None):
        dX, _, _ = fqt.layer_norm_backward(dY, X, mean, rstd, ga)
        _check(dX, X, dY, mean, rstd, ga, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(70, 96), (400, 1024), (9, 8200), (5, 335)])
def test_gradients_into_wider_rows(rows, cols, dtype):
    """dX in columns of wider rows, on 16 bytes and off them; nothing beside it is written."""
    X, dY, mean, rstd, gamma = _case(rows, cols, dtype)
    for left, gap in ((16, 32), (3, 8)):
        wide = torch.full((rows + 1, cols + gap), 5.0, dtype=DTYPES[dtype], device="cuda")
        out = wide[:rows, left:left + cols]
        fqt.layer_norm_backward(dY, X, mean, rstd, gamma, out_x=out)
        _check(out, X, dY, mean, rstd, gamma, dtype)
        assert (wide[rows:] == 5).all()
        assert (wide[:, :left] == 5).all() and (wide[:, left + cols:] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(400, 1024), (50, 9000)])
def test_vectors_off_16_bytes(rows, cols, dtype):
    """Aligned rows beside a scale and a shift that lie one entry into their memory."""
    X, dY, mean, rstd, gamma = _case(rows, cols, dtype)
    ga = torch.cat([gamma[:1], gamma])[1:]
    be = torch.cat([gamma[:1], 0.1 * gamma])[1:]
    assert ga.data_ptr() % 16 == 4 and be.data_ptr() % 16 == 4
    dX, dgamma, dbeta = fqt.layer_norm_backward(dY, X, mean, rstd, ga)
    _check(dX, X, dY, mean, rstd, gamma, dtype)
    xh = (X.double() - mean.double()[:, None]) * rstd.double()[:, None]
    for got, terms in ((dgamma, dY.double() * xh), (dbeta, dY.double())):
        # at most `rows` additions and two roundings of a term
        tol = (rows + 2) * U * terms.abs().sum(0)
        assert ((got.double() - terms.sum(0)).abs() <= tol).all()
    Y, _, _ = fqt.layer_norm_forward(X, ga, be)
    y = xh * gamma.double() + 0.1 * gamma.double()
    # the mean's error, 64 u of the largest entry, and a few roundings
    tol = 1e-5 * y.abs().amax(1, keepdim=True) + ROUND[dtype] * y.abs() + 1e-5
    assert ((Y.double() - y).abs() <= tol).all()
