"""The network's batch normalisation is PyTorch's own, and the rectifiers stand behind it (no GPU: the quantized convolutions are
replaced by PyTorch's)."""
import pytest
import torch

from paper_2310_03675_amd import resnet
from paper_2310_03675_amd.autograd import HdqtConv2d


def _network(**options):
    torch.manual_seed(0)
    net = resnet.ResNet18(**options)
    for m in list(net.modules()):
        for name, conv in list(m.named_children()):
            if isinstance(conv, HdqtConv2d):
                setattr(m, name, torch.nn.Conv2d(conv.weight.shape[0] // conv.k ** 2, conv.weight.shape[1], conv.k, conv.stride, conv.pad, bias=False))
    return net


def _rectified(net, x):
    """What the stem and every block's first half hand on, and what their normalisations give."""
    seen = {}
    hooks = [net.blocks.register_forward_pre_hook(lambda m, a: seen.update(stem=a[0])),
             net.bn0.register_forward_hook(lambda m, a, out: seen.update(bn0=out))]
    for i, block in enumerate(net.blocks):
        hooks += [block.conv_b.register_forward_pre_hook(lambda m, a, i=i: seen.update({f"half{i}": a[0]})),
                  block.bn_a.register_forward_hook(lambda m, a, out, i=i: seen.update({f"bn{i}a": out}))]
    with torch.no_grad():
        out = net(x)
    for h in hooks:
        h.remove()
    return out, seen


@pytest.mark.parametrize("convert", [False, True])
def test_the_rectifier_stays_when_the_normalisation_is_replaced(convert):
    net = _network(head="loss")
    x = torch.randn(4, 3, 32, 32)
    net.train()
    net(x)                                        # (running statistics)
    net.eval()
    want, _ = _rectified(net, x)
    if convert:                                   # the usual step in front of data parallel training
        net = torch.nn.SyncBatchNorm.convert_sync_batchnorm(net).eval()
    got, seen = _rectified(net, x)
    assert torch.equal(got, want)
    for name in ["stem"] + [f"half{i}" for i in range(8)]:
        assert float(seen[name].min()) == 0.0, name
    for name in ["bn0"] + [f"bn{i}a" for i in range(8)]:          # (a hook sees the normalisation alone)
        assert float(seen[name].min()) < 0.0, name


def test_a_target_needs_the_loss_head():
    """Refused before anything runs: the quantized classifier has no loss, and logits are not what a caller with targets
    asks for."""
    net = _network()
    net.fc = torch.nn.Linear(512, 100)
    x = torch.zeros(2, 3, 32, 32)
    assert tuple(net(x).shape) == (2, 100)
    with pytest.raises(ValueError):
        net(x, torch.zeros(2, dtype=torch.int64))
