"""What clip_gradients hands on (no GPU: the library's call is replaced)."""
import torch

from paper_2310_03675_amd import autograd as A


def test_without_gradients_the_norm_is_on_the_parameters_device():
    """As the norm is that there is with gradients, so that a training loop may add either up."""
    p = torch.nn.Parameter(torch.zeros(2, device="meta"))
    for parameters in ([p], (p for _ in range(2))):
        norm = A.clip_gradients(parameters, 1.0)
        assert norm.device.type == "meta" and norm.shape == () and norm.dtype == torch.float32
    assert float(A.clip_gradients([], 1.0)) == 0.0


def test_a_single_tensor(monkeypatch):
    """A parameter is its own list: its rows have no gradients, and nothing was clipped."""
    got = []
    monkeypatch.setattr(A.B, "clip_grad_norm", lambda grads, *how: got.append((grads, how)) or torch.ones(()))
    p = torch.nn.Parameter(torch.zeros(4, 3))
    p.grad = torch.ones(4, 3)
    assert float(A.clip_gradients(p, 0.5, 2.0, 1e-6)) == 1.0
    assert len(got) == 1 and got[0][0][0] is p.grad and len(got[0][0]) == 1 and got[0][1] == (0.5, 2.0, 1e-6)
