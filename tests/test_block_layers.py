"""The adapters' module and the quantized layer beside them, without a GPU."""
import pytest
import torch

from paper_2310_03675_amd import autograd as A


def test_a_layer_with_adapters_asks_for_ids():
    """Left out, the adapters would not be used, nor trained."""
    layer = A.HdqtLinear(8, 8, adapters=A.Adapters(8, 8, 2, 4))
    for m in (layer, layer.eval()):
        with pytest.raises(ValueError, match="asks for ids"):
            m(torch.zeros(2, 8))
