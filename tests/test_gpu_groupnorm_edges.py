"""Group normalisation at the edges of its rules, against 64 bits.  Tolerances as in test_gpu_groupnorm.py: 2^-8 for one rounding
to bfloat16 and 2e-6 of the 2-norm for what is done in 32 bits."""
import pytest
import torch

from paper_2310_03675_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def near(got, want, tol, norm=None):
    d, n = (got.double().cpu().reshape(want.shape) - want).norm(), want.norm() if norm is None else norm
    assert d <= tol * n + 1e-30, (float(d / n), tol)


def rows_of(x, dy, G, eps=1e-5):
    """Outputs in 64 bits of images x [n, P, C] without parameters or activation, and the first term of dx."""
    n, P, C = x.shape
    v, d = (t.double().cpu().reshape(n, P, G, C // G) for t in (x, dy))
    mu = v.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt((v - mu).square().mean((1, 3), keepdim=True) + eps)
    xh = (v - mu) * rstd
    dx = rstd * (d - d.mean((1, 3), keepdim=True) - xh * (d * xh).mean((1, 3), keepdim=True))
    return xh.reshape(n, P, C), dx.reshape(n, P, C), (rstd * d).norm()


def test_more_groups_than_a_launch_has_threads_for():
    """Groups of 520 channels, 4.3 million of them: a workgroup of 1024 threads each would be more than 32 bits count."""
    images, C, G = 65535, 33800, 65
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty(images, 1, C, dtype=BF16, device="cuda").normal_(0.3, 1.5, generator=g)
    dy = torch.empty_like(x).normal_(generator=g)
    y, saved = B.groupnorm_fwd(x, G)
    dx, _, db = B.groupnorm_bwd(dy, x, saved, G)
    some = torch.tensor([0, 1, 32767, 32768, 65533, 65534], device="cuda")
    want, dwant, terms = rows_of(x[some], dy[some], G)
    near(y[some], want, 2.0 ** -8 + 2e-6)
    near(dx[some], dwant, 2.0 ** -8 + 2e-6, norm=terms)
    for c in (0, 519, C - 1):                # sums of 65535 terms, added up in 64 bits
        near(db[c], dy[:, 0, c].double().sum().cpu(), 1.0, norm=2e-6 * dy[:, 0, c].double().norm().cpu() + 2.0 ** -23 * db[c].abs().cpu())
