"""A residual block whose forward pass the backward pass makes again."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2310_03675_amd import autograd as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("reentrant", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_checkpointed_block_is_the_block(reentrant, dtype):
    """Two blocks of dropout, normalisation and adapters, of the same layers, step after step: outputs have the bits that they have without
    checkpointing, and gradients are the same but for the order in which autograd adds up what reaches one tensor.

    That order: each block's input is given to it twice and used three times, so that two additions to a block are associated in
    one way or the other, and a parameter's two parts meet in either order; half a step each (`eps / 2` of the terms), on both sides, and
    through the block before: 2 x 2 x 2 of them and as many again for the backward calls' own roundings of what they are given, 16."""
    torch.manual_seed(3)
    drop, norm = A.ResidualDropout(0.2, seed=1, layer_id=1), A.ResidualNorm(72, p=0.3, seed=1, layer_id=2, device="cuda")
    bank = A.Adapters(72, 72, 3, 4, device="cuda").to(dtype)
    torch.nn.init.normal_(bank.B, std=0.1)
    ids = torch.randint(-1, 3, (90,), device="cuda")

    def block(x, total):
        y, s = norm(bank(x, drop(x, total), ids), total)
        return y, s

    def network(x, wrap):
        y, s = wrap(block, x, x)
        y, s = wrap(block, y, s)
        return wrap(drop, y, s)

    params = [norm.weight, norm.bias, bank.A, bank.B]

    def steps(wrap):
        drop.masks.step = norm.masks.step = 0
        got = []
        for k in range(3):
            x = torch.randn(90, 72, generator=torch.Generator().manual_seed(k)).to(dtype).cuda().requires_grad_()
            for t in params:
                t.grad = None
            out = network(x, wrap)
            (out.float() ** 2).sum().backward()
            got.append([out.detach(), x.grad] + [t.grad for t in params])
        assert drop.masks.step == 9 and norm.masks.step == 6
        return got

    plain = steps(lambda f, *a: f(*a))
    again = steps(lambda f, *a: checkpoint(f, *a, use_reentrant=reentrant))
    for one, other in zip(plain, again):
        assert torch.equal(one[0], other[0])
        for p, q in zip(one[1:], other[1:]):
            assert float((p - q).double().norm()) <= 16 * torch.finfo(dtype).eps / 2 * float(p.double().norm())
