"""The classifier's loss at the edges of its rules, against 64 bits.  Tolerances as in test_gpu_xent.py."""
import math

import pytest
import torch

from paper_2310_03675_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
IGNORE = -100


def near(got, want, tol, floor=0.0):
    d = float((got.double().to(want.device) - want).norm())
    assert d <= tol * max(float(want.norm()), floor) + 1e-12, (d / (float(want.norm()) + 1e-300), tol)


def test_rows_that_are_packed_one_after_the_other():
    """34 GB of features whose rows are no whole 16 bytes: more than one launch packs."""
    M, K, N = 4194240, 4105, 3
    X = torch.empty(M, K, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(0))
    g = torch.Generator().manual_seed(1)
    W = (torch.randn(K, N, generator=g) * 1.5 / math.sqrt(K)).to(BF16).cuda()
    t = torch.randint(0, N, (M,), generator=g).cuda()
    loss, _ = B.xent_fwd(X, W, t, reduction="none")
    for part in (slice(0, 4000), slice(M // 2 - 2000, M // 2 + 2000), slice(3728000, 3732000), slice(M - 4000, M)):
        z = X[part].double().cpu() @ W.double().cpu()
        want = torch.nn.functional.cross_entropy(z, t[part].cpu(), reduction="none")
        near(loss[part], want, 4e-5, floor=math.sqrt(4000))
