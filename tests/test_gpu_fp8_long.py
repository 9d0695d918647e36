"""FP8 products over long contractions whose terms have one sign, where what the tensor
cores drop adds up instead of cancelling.

Tolerances.  A step of 32 terms drops less than 2^-23 of the accumulator (all magnitudes
so far, at most those of its own terms).  With A terms to an accumulator that is
A / 32 2^-23 of the sum of magnitudes S; the accumulators are then added in fp32, each
addition off by 2^-24 of at most S, those of the up to 8 CTAs that share a tile too:
|error| <= ((A / 32) 2^-23 + (K / A + 8) 2^-24) S, with A = 1024 for an fp32 output and
8192 for a bf16 one, which adds a rounding, at most 2^-8 of the result.
"""
import pytest
import torch

from paper_2010_14298_gb300 import fqt

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def _rows(rows, K, seed, first=0.0):
    """rows x K positive entries, every row of a size of its own, the first 64 entries
    of a row larger by `first` times the rest's sum."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.rand(rows, K, generator=g, device="cuda").mul_(0.5).add_(0.5)
    x *= 1 + torch.arange(rows, device="cuda")[:, None] / rows
    if first:
        x[:, :64] *= first * K / 64
    return x


def _bound(K, per):
    return min(K, per) / 32 * 2.0 ** -23 + (-(-K // per) + 8) * 2.0 ** -24


# tiles of pairs, of single CTAs, and shared by clusters
@pytest.mark.parametrize("first", [0.0, 2.0])
@pytest.mark.parametrize("M,N,K", [(2048, 2048, 16384), (2048, 2048, 65536), (1280, 1280, 65536),
                                   (40, 5000, 65536), (128, 256, 524288)])
def test_fp32_outputs_of_one_sign(M, N, K, first):
    a, _ = fqt.quantize_fp8(_rows(M, K, 1, first))
    b, _ = fqt.quantize_fp8(_rows(N, K, 2))
    want = a.dequantize().double() @ b.dequantize().double().t()
    out = fqt.fp8_matmul(a, b)
    assert ((out.double() / want - 1).abs() <= _bound(K, 1024)).all()


def _repeated(q, times):
    """q's rows, all of them that many times."""
    return fqt.Fp8Tensor(q.codes.repeat(times, 1), q.scales.repeat(1, times, 1), q.rows * times,
                         q.cols)


# tiles of pairs, and shared by clusters (whose CTAs add an eighth of K each)
@pytest.mark.parametrize("first", [0.0, 2.0])
@pytest.mark.parametrize("M,N,K", [(2048, 2048, 1 << 21), (256, 256, 1 << 22)])
def test_bf16_outputs_of_one_sign(M, N, K, first):
    """An output alone shows its rounding first, so the mean over 256 x 256 different ones
    is held to the bound too: roundings to nearest of values that fill a binade have a
    standard deviation of at most 2^-8 / sqrt(3), their mean a 256th of that, times 4."""
    a, _ = fqt.quantize_fp8(_rows(256, K, 1, first).bfloat16())
    b, _ = fqt.quantize_fp8(_rows(256, K, 2).bfloat16())
    want = sum(p.dequantize().double() @ q.dequantize().double().t() for p, q in _slices(a, b))
    out = fqt.fp8_matmul(_repeated(a, M // 256), _repeated(b, N // 256), dtype=torch.bfloat16)
    off = out.double() / want.repeat(M // 256, N // 256) - 1
    assert (off.abs() <= 2.0 ** -8 + _bound(K, 8192)).all()
    assert abs(float(off[:256, :256].mean())) <= _bound(K, 8192) + 4 * 2.0 ** -8 / 3 ** 0.5 / 256


def _slices(a, b, step=1 << 18):
    """The two matrices' columns in parts (64 bits of all of them take too much room)."""
    for k in range(0, a.cols, step):
        yield [fqt.Fp8Tensor(q.codes[:, k:k + step].contiguous(),
                             q.scales[k // 512:(k + step) // 512].contiguous(), q.rows, step)
               for q in (a, b)]
