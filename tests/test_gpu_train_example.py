"""The operators around the products as modules, against PyTorch's in 64 bits, and the training example that runs them with the
quantized layers.

Tolerances: those of the operators' own tests (2e-6 normalised, 1e-5 the loss and its gradients in fp32, of the
2-norm)."""
import math

import pytest
import torch

from paper_2310_03675_amd import autograd as A
from paper_2310_03675_amd import resnet, train

pytestmark = pytest.mark.gpu


def near(got, want, tol):
    assert float((got.double().cpu() - want).norm()) <= tol * float(want.norm()) + 1e-12


@pytest.mark.parametrize("innermost", [True, False])
def test_group_norm_module(innermost):
    torch.manual_seed(0)
    m = A.GroupNormAct(4, 24, act="silu", device="cuda")
    torch.nn.init.normal_(m.weight, 1.0, 0.2)
    torch.nn.init.normal_(m.bias, 0.0, 0.2)
    x = torch.randn(3, 24, 9, 7, device="cuda")
    if innermost:
        x = x.contiguous(memory_format=torch.channels_last)
    x.requires_grad_()
    y = m(x)
    r = torch.randn(3, 24, 9, 7, generator=torch.Generator().manual_seed(1)).cuda()
    (y * r).sum().backward()
    xd, w, b = (v.detach().double().cpu().requires_grad_() for v in (x, m.weight, m.bias))
    want = torch.nn.functional.silu(torch.nn.functional.group_norm(xd, 4, w, b, 1e-5))
    (want * r.double().cpu()).sum().backward()
    near(y.detach(), want.detach(), 2e-6)
    for got, of in ((x.grad, xd.grad), (m.weight.grad, w.grad), (m.bias.grad, b.grad)):
        near(got, of, 2e-5)
    with pytest.raises(ValueError):
        A.GroupNormAct(5, 24)


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_classifier_with_classes_to_come(reduction):
    torch.manual_seed(0)
    m = A.ClassifierLoss(40, 60, classes=35, reduction=reduction, device="cuda")
    torch.nn.init.normal_(m.bias)
    x = torch.randn(5, 8, 40, device="cuda", requires_grad=True)
    t = torch.randint(0, 35, (5, 8), device="cuda")
    t[2, 3] = -100
    loss = m(x, t)
    (loss * 2).sum().backward()
    xd, w, b = (v.detach().double().cpu().requires_grad_() for v in (x, m.weight, m.bias))
    z = xd.reshape(-1, 40) @ w[:, :35] + b[:35]
    want = torch.nn.functional.cross_entropy(z, t.cpu().reshape(-1), reduction=reduction)
    (want * 2).sum().backward()
    near(loss.detach(), want.detach(), 1e-5)
    for got, of in ((x.grad, xd.grad), (m.weight.grad, w.grad), (m.bias.grad, b.grad)):
        near(got, of, 1e-5)
    assert not m.weight.grad[:, 35:].any()                      # (classes that are not in use)
    near(m.logits(x.detach()).reshape(-1, 35), z.detach(), 1e-5)
    # a part of the gradients
    m.weight.requires_grad_(False)
    x.grad = None
    m(x, t).sum().backward()
    assert x.grad is not None


def test_clip_gradients():
    ps = [torch.nn.Parameter(torch.randn(9, 5, device="cuda")) for _ in range(3)] + [torch.nn.Parameter(torch.zeros(2, device="cuda"))]
    for p in ps[:3]:
        p.grad = torch.randn_like(p)
    want = torch.stack([p.grad.double().norm() for p in ps[:3]]).norm()
    before = [p.grad.clone() for p in ps[:3]]
    norm = A.clip_gradients(ps, 0.5)
    assert float(norm) == pytest.approx(float(want), rel=1e-6)
    for p, g in zip(ps, before):
        near(p.grad, g.double().cpu() * (0.5 / (float(want) + 1e-6)), 1e-6)
    assert float(A.clip_gradients([ps[3]], 1.0)) == 0.0


def test_training_example():
    said = []
    history = train.train(tasks=2, steps=10, batch=64, report=said.append)
    assert len(history) == 20 and len(said) == 2
    assert all(math.isfinite(a) and math.isfinite(b) and b > 0 for a, b in history)
    first, second = [a for a, _ in history[:10]], [a for a, _ in history[10:]]
    assert abs(first[0] - math.log(50)) < 1.5                    # (50 classes, nothing learnt)
    assert min(first[-3:]) < first[0] and min(second[-3:]) < second[0]
    with pytest.raises(ValueError):
        train.train(tasks=3, classes=100)
    with pytest.raises(ValueError):
        resnet.ResNet18(norm="layer")
