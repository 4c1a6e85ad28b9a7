"""A residual block's operators as modules, together with the quantized layer they stand around.

Tolerances: those of the operators' own tests, 2e-6 of the terms and, through several of them one after the other, their sum."""
import pytest
import torch

from paper_2310_03675_amd import autograd as A
from paper_2310_03675_amd import binding as B
from residual_block import adapters, dropped, kept, layer_norm, rate

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def near(got, want, tol):
    assert float((got.detach().double().cpu() - want).norm()) <= tol * float(want.norm()) + 1e-12


def test_residual_dropout_module():
    m = A.ResidualDropout(0.3, seed=5, layer_id=2)
    x, r = (torch.randn(6, 4, 33, device="cuda", requires_grad=True) for _ in range(2))
    g = torch.randn(6, 4, 33, device="cuda")
    for step in range(2):
        x.grad = r.grad = None
        y = m(x, r)
        (y * g).sum().backward()
        d = B.Dropout(0.3, 5 + step, 2)
        near(y, r.detach().double().cpu() + dropped(x.detach(), d), 1e-6)
        near(x.grad, dropped(g, d), 1e-6)
        assert torch.equal(r.grad, g)
    near(m(x), dropped(x.detach(), B.Dropout(0.3, 7, 2)), 1e-6)
    m.eval()
    assert torch.equal(m(x, r), r + x) and m(x) is x
    # inputs that are not dense in order, and one that needs no gradient
    m.train()
    t = x.detach().transpose(0, 1)
    assert torch.equal(m(t), B.dropout(t.contiguous(), B.Dropout(0.3, 8, 2)))


def test_a_step_that_moved_is_noticed():
    m = A.ResidualDropout(0.5)
    m.masks.counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    x = torch.randn(100, device="cuda", requires_grad=True)
    y = m(x)
    m.masks.counter.add_(1)
    with pytest.raises(RuntimeError):
        y.sum().backward()


@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_residual_norm_module(p, dtype):
    torch.manual_seed(0)
    m = A.ResidualNorm(72, p=p, seed=3, layer_id=4, device="cuda")
    torch.nn.init.normal_(m.weight, 1.0, 0.2)
    torch.nn.init.normal_(m.bias, 0.0, 0.2)
    x, r = (torch.randn(5, 9, 72, device="cuda").to(dtype).requires_grad_() for _ in range(2))
    gy, gs = (torch.randn(5, 9, 72, device="cuda").to(dtype) for _ in range(2))
    y, s = m(x, r)
    torch.autograd.backward((y, s), (gy, gs))
    d = B.Dropout(p, 3, 4) if p else None
    want = layer_norm(x.detach(), gy, m.weight.detach(), m.bias.detach(), r.detach(), gs, d, held=s.detach())
    tol = 4e-6 if dtype == F32 else 4e-6 + 2.0 ** -8
    for got, of in ((y, "y"), (s, "sum"), (x.grad, "dx"), (r.grad, "dresidual")):
        near(got, want[of], tol)
    near(m.weight.grad, want["dweight"], 2e-5)
    near(m.bias.grad, want["dbias"], 2e-5)
    # only one of the two outputs is used
    for which, grads in ((0, (gy, None)), (1, (None, gs))):
        x.grad = r.grad = m.weight.grad = None
        m.masks.step = 0
        m(x, r)[which].backward(grads[which])
        one = layer_norm(x.detach(), gy if which == 0 else torch.zeros_like(gy), m.weight.detach(), None, r.detach(), grads[1], d, held=s.detach())
        near(x.grad, one["dx"], tol)
        near(r.grad, one["dresidual"], tol)
        assert (m.weight.grad is None) == (which == 1)
    # without a residual
    m.masks.step = 0
    y = m(x)
    near(y, layer_norm(x.detach(), gy, m.weight.detach(), m.bias.detach(), None, None, d)["y"], tol + (2.0 ** -8 if dtype == BF16 else 0))
    m.eval()
    y, s = m(x, r)
    near(s, r.detach().double().cpu() + x.detach().double().cpu(), tol)


def test_adapters_module():
    torch.manual_seed(0)
    m = A.Adapters(40, 56, 5, 4, alpha=8.0, device="cuda")
    x, base = torch.randn(3, 7, 40, device="cuda", requires_grad=True), torch.randn(3, 7, 56, device="cuda", requires_grad=True)
    ids = torch.randint(-1, 5, (3, 7), device="cuda")
    assert torch.equal(m(x, base, ids), base)                      # (B is zero)
    torch.nn.init.normal_(m.B)
    g = torch.randn(3, 7, 56, device="cuda")
    out = m(x, base, ids)
    (out * g).sum().backward()
    scale = torch.full((5,), 2.0)
    want = adapters(x.detach().reshape(21, 40), m.A.detach(), m.B.detach(), ids.reshape(21), scale, base.detach().reshape(21, 56), g.reshape(21, 56))
    near(out.reshape(21, 56), want["out"], 1e-5)
    near(x.grad.reshape(21, 40), want["dx"], 1e-5)
    near(m.A.grad, want["dA"], 1e-5)
    near(m.B.grad, want["dB"], 1e-5)
    assert torch.equal(base.grad, g)
    # a frozen bank, and an input without a gradient
    m.requires_grad_(False)
    base.grad = None
    m(x.detach(), base, ids).sum().backward()
    assert torch.equal(base.grad, torch.ones_like(base))


class Block(torch.nn.Module):
    """y = norm(residual + dropout(quantized layer with adapters(x)))."""

    def __init__(self, width, tasks, p):
        super().__init__()
        self.layer = A.HdqtLinear(width, width, cfg=A.LayerConfig(had_block=16), device="cuda", adapters=A.Adapters(width, width, tasks, 4, device="cuda"))
        self.norm = A.ResidualNorm(width, p=p, seed=9, layer_id=1, device="cuda")

    def forward(self, x, ids):
        return self.norm(self.layer(x, ids), x)


def test_a_block_of_all_of_them():
    """Two blocks in training: the loss's gradients of adapters and norms against 64 bits, the quantized products' results taken as
    they were (their own gradients are other tests')."""
    torch.manual_seed(1)
    width, M, tasks, p = 64, 96, 3, 0.1
    block = Block(width, tasks, p).train()
    torch.nn.init.normal_(block.layer.adapters.B, std=0.1)
    block.layer.weight.requires_grad_(False)
    cap = {}
    block.layer.cfg.capture = cap
    x = torch.randn(M, width, device="cuda")
    ids = torch.randint(-1, tasks, (M,), device="cuda")
    gy, gs = torch.randn(M, width, device="cuda"), torch.randn(M, width, device="cuda")
    y, s = block(x, ids)
    torch.autograd.backward((y, s), (gy, gs))
    a = block.layer.adapters
    z = cap["Z"] + block.layer.bias.detach()
    fwd = adapters(x, a.A.detach(), a.B.detach(), ids, a.scale, z)
    d = B.Dropout(p, 9, 1)
    mask = kept(M * width, p, 9, 1).reshape(M, width)
    total = x.double().cpu() + torch.where(mask, fwd["out"] * rate(p), torch.zeros((), dtype=torch.float64))
    near(s, total, 4e-6)
    want = layer_norm(x, gy, block.norm.weight.detach(), block.norm.bias.detach(), None, gs, None, held=s.detach())
    near(y, want["y"], 4e-6)
    near(block.norm.weight.grad, want["dweight"], 2e-5)
    dz = torch.where(mask, want["dresidual"] * rate(p), torch.zeros((), dtype=torch.float64))
    back = adapters(x, a.A.detach(), a.B.detach(), ids, a.scale, None, dz)
    near(a.A.grad, back["dA"], 2e-5)
    near(a.B.grad, back["dB"], 2e-5)
    near(block.layer.bias.grad, dz.sum(0), 2e-5)


def test_a_captured_block():
    """Forward and backward in one graph, with the step's counter: every replay is the eager step of that count."""
    torch.manual_seed(2)
    norm, bank = A.ResidualNorm(48, p=0.3, seed=2, layer_id=6, device="cuda"), A.Adapters(48, 48, 3, 4, device="cuda")
    torch.nn.init.normal_(bank.B, std=0.1)
    norm.masks.counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    x, ids = torch.randn(200, 48, device="cuda"), torch.randint(-1, 3, (200,), device="cuda")
    params = list(norm.parameters()) + [bank.A, bank.B]

    def step():
        y, s = norm(bank(x, x, ids), x)
        return (y.detach(), s.detach()) + torch.autograd.grad((y * y).sum() + s.sum(), params)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in (3, 0, 7):
        norm.masks.counter.fill_(k)
        x.mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in got]
        assert all(torch.equal(p, q) for p, q in zip(held, step()))
