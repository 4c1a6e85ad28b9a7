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
