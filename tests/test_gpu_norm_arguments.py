"""What dora_residual_norm_backward asks of a branch whose gradient is dx itself."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
def test_branch_without_parameters(gpu, monkeypatch, native):
    """a is not read there, but its gradient has to have its sizes and type."""
    if not native:
        for name in ("_native_call", "_native_vectors", "_native_describe", "_native_written"):
            monkeypatch.setattr(gpu, name, gpu._leave_to_ctypes)
    h, w = torch.randn((6, 64), device="cuda"), torch.ones(64, device="cuda")
    for scale in (None, w):                 # with a scale, where a is read, the same errors
        for a, error, text in ((h[:5], gpu.DoraError, "shape"), (torch.zeros((6, 32), device="cuda"), gpu.DoraError, "shape"),
                               (h.bfloat16(), gpu.DoraError, "dtype"), (h.view(6, 2, 32), gpu.DoraError, "shape"),
                               (h.half(), TypeError, ""), (h.cpu(), ValueError, ""), (h.view(-1), ValueError, ""),
                               (h.tolist(), TypeError, "")):
            with pytest.raises(error, match=f"(?i){text}"):
                gpu.dora_residual_norm_backward(h, h, a, w, scale=scale)
    got = gpu.dora_residual_norm_backward(h, h, h, w)
    assert got.da is got.dx
    a = h.clone()
    again = gpu.dora_residual_norm_backward(h, h, a, w, dx=a)          # in a's place
    assert again.dx is a and torch.equal(a, got.dx)
