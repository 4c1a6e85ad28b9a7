"""Low-rank adapters on inputs whose results have no rounding, or one that the test is about."""
import pytest
import torch

from paper_2310_03675_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("r", [8, 24, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M, K", [(33, 4133), (700, 2080), (4200, 2080)])
def test_every_step_of_a_contraction_counts(M, K, r, dtype):
    """Whole numbers, so that every result is exact: a wave takes several steps one after the other through the same LDS, the last of
    them no whole one.  Sums stay under 256, to where bfloat16 holds every whole number."""
    g = torch.Generator().manual_seed(M + r)
    n, N = 3, 264
    whole = lambda *s: torch.randint(-3, 4, s, generator=g).double()
    few = lambda *s: torch.randint(-1, 2, s, generator=g).double() * (torch.rand(s, generator=g) < 1 / 16)
    x, A, ids = whole(M, K), few(n, K, r), torch.randint(-1, n, (M,), generator=g)
    # a rank's value comes out in column rank, and as its negative in the last ones
    Bm = torch.zeros(n, r, N, dtype=torch.float64)
    for rank in range(r):
        Bm[:, rank, rank] = 1
        Bm[:, rank, N - 1 - rank] = -1
    h = torch.zeros(M, r, dtype=torch.float64)
    for a in range(n):
        h[ids == a] = x[ids == a] @ A[a]
    assert 10 < float(h.abs().max()) <= 256
    want = torch.zeros(M, N, dtype=torch.float64)
    want[:, :r] += h
    want[:, N - r:] -= h.flip(1)
    dev = lambda t: t.to(dtype).cuda()
    out, _ = B.adapters_fwd(dev(x), dev(A), dev(Bm), ids.cuda())
    assert torch.equal(out.double().cpu(), want)
    # the same way round for the gradient: dx = (dy B^T) A^T with B in A's place
    Bw, Aw = A.transpose(1, 2).contiguous(), Bm.transpose(1, 2).contiguous()
    x0 = torch.zeros(M, N, dtype=torch.float64)
    _, saved = B.adapters_fwd(dev(x0), dev(Aw), dev(Bw), ids.cuda())
    dx, dA, dB = B.adapters_bwd(dev(x), dev(x0), dev(Aw), dev(Bw), ids.cuda(), saved)
    assert torch.equal(dx.double().cpu(), want) and not dA.any() and not dB.any()
