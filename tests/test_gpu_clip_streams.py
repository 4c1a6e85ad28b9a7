"""The gradients' norm and their clipping on a stream that is not the default one."""
import math

import pytest
import torch

from paper_2310_03675_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [2.0, math.inf])
@pytest.mark.parametrize("lengths", [(300, 70001, 5), (9_000_000, 8_000_001)])      # (the product's workgroups add up themselves; a launch does)
def test_calls_on_a_side_stream(kind, lengths):
    """The default stream's results, of what was written on the side stream before."""
    g = torch.Generator(device="cuda").manual_seed(4)
    grads = [torch.randn(n, generator=g, device="cuda").to(dtype) for n, dtype in zip(lengths, (torch.float32, torch.bfloat16, torch.float32))]
    want = [torch.empty_like(v) for v in grads]
    norm0 = B.clip_grad_norm(grads, 0.1, norm_type=kind, out=want)
    late, out = [torch.zeros_like(v) for v in grads], [torch.zeros_like(v) for v in grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a, b in zip(late, grads):
            a.copy_(b)
    alone = B.grad_norm(late, kind, stream=side)
    norm = B.clip_grad_norm(late, 0.1, norm_type=kind, out=out, stream=side)
    here = B.clip_grad_norm(late, 0.1, norm_type=kind, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(norm, norm0) and torch.equal(alone, norm0) and torch.equal(here, norm0)
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, out, late))
    torch.cuda.synchronize()
