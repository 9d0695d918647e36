"""The calls of a training step around the quantized layers refuse tensors and workspaces
that are not on their first tensor's GPU, before a kernel gets an address."""
import pytest
import torch

from paper_2010_14298_gb300 import fqt


class _Elsewhere:
    """A float32 tensor on GPU 1 as far as a check asks."""
    dtype, device = torch.float32, torch.device("cuda", 1)
    is_cuda = True
    shape = torch.Size((4, 64))

    def get_device(self):
        return 1

    def dim(self):
        return 2

    def numel(self):
        return 256

    def is_contiguous(self):
        return True


def test_other_gpus_are_refused():
    t = _Elsewhere()
    assert fqt._vector(t, "gamma", 256, 1) is t
    assert fqt._rows_in(t, "X", None) == (t, 4, 64, 64, 1)
    assert fqt._rows_out(t, "out", 4, 64, t.dtype, 1, t, None) == (t, 64)
    ws = fqt.Workspace.of_size(256, "cpu")
    ws.buf = t
    assert fqt._scratch(ws, 1) == (t, 256)
    q = fqt.Fp8Tensor.empty(4, 64, device="cpu")
    q.codes = t
    for bad in (lambda: fqt._vector(t, "gamma", 256, 0),
                lambda: fqt._rows_out(t, "out", 4, 64, t.dtype, 0, t, None),
                lambda: fqt._fp8_out(q, "q", 4, 64, 1, 0, t, None),
                lambda: fqt._scratch(ws, 0)):
        with pytest.raises(ValueError, match="GPU 0"):
            bad()


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")
def test_host_tensors_are_refused():
    X = torch.ones((4, 64), device="cuda")
    v, m = torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    ws = fqt.Workspace.of_size(1 << 20, "cpu")
    q, _ = fqt.quantize_fp8(X)
    host = fqt.Fp8Tensor.empty(4, 64, device="cpu")
    for bad in (lambda: fqt.layer_norm_forward(X, v.cpu()),
                lambda: fqt.layer_norm_forward(X, v, v.cpu()),
                lambda: fqt.layer_norm_forward(X, out=X.cpu()),
                lambda: fqt.layer_norm_forward(X, mean=m.cpu()),
                lambda: fqt.layer_norm_forward(X, rstd=m.cpu()),
                lambda: fqt.layer_norm_backward(X.cpu(), X, m, m),
                lambda: fqt.layer_norm_backward(X, X, m.cpu(), m),
                lambda: fqt.layer_norm_backward(X, X, m, m.cpu()),
                lambda: fqt.layer_norm_backward(X, X, m, m, v.cpu()),
                lambda: fqt.layer_norm_backward(X, X, m, m, out_x=X.cpu()),
                lambda: fqt.layer_norm_backward(X, X, m, m, out_gamma=v.cpu()),
                lambda: fqt.layer_norm_backward(X, X, m, m, out_beta=v.cpu()),
                lambda: fqt.layer_norm_backward(X, X, m, m, ws=ws),
                lambda: fqt.quantize_fp8(X, q=host), lambda: fqt.quantize_fp8(X, qt=host),
                lambda: fqt.quantize_fp8(X, ws=ws),
                lambda: fqt.fp8_matmul(q, host), lambda: fqt.fp8_matmul(host, q),
                lambda: fqt.fp8_matmul(q, q, out=torch.ones((4, 4))),
                lambda: fqt.fp8_matmul(q, q, ws=ws),
                lambda: fqt.clip_grad_norm([X], 1.0, ws=ws),
                lambda: fqt.grad_norm([X], norm=torch.ones(1)),
                lambda: fqt.grad_norm([X], ws=ws)):
        with pytest.raises(ValueError):
            bad()
    torch.cuda.synchronize()
    assert (X == 1).all()
