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


@pytest.mark.parametrize("into", [lambda m: m.to(torch.bfloat16), lambda m: m.bfloat16(), lambda m: m.double(),
                                  lambda m: torch.nn.Sequential(m).to("cpu", torch.bfloat16)[0], lambda m: m.to("meta").to(torch.bfloat16)])
def test_the_scales_of_adapters_stay_in_32_bits(into):
    m = A.Adapters(8, 8, 3, 24, alpha=16.0)
    scale = m.scale.clone()
    m = into(m)
    assert m.scale.dtype == torch.float32 and m.A.dtype != torch.float32 and set(m.state_dict()) == {"A", "B", "scale"}
    assert m.scale.is_meta or torch.equal(m.scale, scale)
