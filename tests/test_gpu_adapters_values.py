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


@pytest.mark.parametrize("r", [3, 4, 5, 6, 7, 9, 18, 30, 33, 66, 127])
@pytest.mark.parametrize("M", [20, 300])
def test_an_infinity_in_a_matrix_gives_infinities(M, r):
    """fp32: dx and out have the formula's infinities, with their signs, where it has them, and the same bits everywhere else."""
    g = torch.Generator().manual_seed(r)
    K, N, n = 70, 140, 2
    f = lambda *s: torch.randn(*s, generator=g).cuda()
    x, dy, base, A, Bm = f(M, K), f(M, N), f(M, N), f(n, K, r), f(n, r, N)
    ids = torch.randint(0, n, (M,), generator=g).cuda()
    out0, saved0 = B.adapters_fwd(x, A, Bm, ids, base=base)
    dx0 = B.adapters_bwd(dy, x, A, Bm, ids, saved0, need=(True, False, False))[0]
    h = torch.stack([x[i].double() @ A[ids[i]].double() for i in range(M)])
    back = torch.stack([dy[i].double() @ Bm[ids[i]].double().t() for i in range(M)])
    for rank in {0, r // 2, max(r - 2, 0), r - 1}:
        infinite = A.clone()
        infinite[1, 33, rank] = float("inf")
        dx = B.adapters_bwd(dy, x, infinite, Bm, ids, saved0, need=(True, False, False))[0]
        want = dx0.clone()
        want[ids == 1, 33] = float("inf") * back[ids == 1, rank].sign().float()
        assert torch.equal(dx, want), rank
        infinite = Bm.clone()
        infinite[1, rank, 77] = float("inf")
        out, _ = B.adapters_fwd(x, A, infinite, ids, base=base)
        want = out0.clone()
        want[ids == 1, 77] = float("inf") * h[ids == 1, rank].sign().float()
        assert torch.equal(out, want), rank


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 5, 70, 200])
def test_an_infinite_scale_of_an_adapter_of_few_rows(rows, dtype):
    """Its gradients are infinite, also where they are added up over parts of the rows of which some have none of its."""
    g = torch.Generator().manual_seed(rows)
    M, K, N, r, n = 1100, 64, 72, 4, 2
    f = lambda *s: (torch.rand(*s, generator=g) + 0.5).to(dtype).cuda()
    x, dy, A, Bm, scale = f(M, K), f(M, N), f(n, K, r), f(n, r, N), torch.tensor([1.0, float("inf")], device="cuda")
    ids = torch.zeros(M, dtype=torch.int64)
    ids[torch.randperm(M, generator=g)[:rows]] = 1
    ids = ids.cuda()
    out, saved = B.adapters_fwd(x, A, Bm, ids, scale)
    dx, dA, dB = B.adapters_bwd(dy, x, A, Bm, ids, saved, scale)
    for t in (out[ids == 1], dx[ids == 1], dA[1], dB[1]):
        assert bool((t == float("inf")).all())
    for t in (out[ids == 0], dx[ids == 0], dA[0], dB[0]):
        assert bool(t.isfinite().all())


LOW = [(6, 64, 128, 5, 2), (20, 20, 24, 9, 2), (20, 24, 20, 40, 2), (40, 4096, 4096, 16, 3), (40, 4096, 4096, 40, 3), (200, 512, 640, 12, 4),
       (700, 130, 200, 16, 3), (700, 130, 200, 33, 3), (700, 131, 203, 60, 3), (700, 130, 200, 128, 2), (6000, 600, 520, 8, 1), (6000, 600, 520, 24, 1)]


@pytest.mark.parametrize("size", LOW, ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_h_has_beyond_one_bfloat16_value(size, dtype):
    """h and g are 1 + k / 1024 or its negative, k from 1 to 6: as one bfloat16 value of eight bits, 1.  What the ones give is cancelled, by the
    base or by another row, and what is left is exact: multiples of 1 / 1024 below 256 of them."""
    M, K, N, r, n = size
    g = torch.Generator().manual_seed(M + r)
    whole = lambda *s: torch.randint(-1, 2, s, generator=g).double()
    ids = torch.randint(0, n, (M // 2,), generator=g).repeat_interleave(2)
    dev = lambda t: t.to(dtype).cuda()
    m = torch.tensor([1.0, 2.0]).double()[torch.randint(0, 2, (M,), generator=g)]

    def split(features):
        """Rows of two values, and matrices that make 1 + k / 1024 of them: the rows, the matrices, the products' ones and what is beyond."""
        v, one, k = torch.zeros(M, features, dtype=torch.float64), torch.ones(n, r).double(), torch.randint(1, 4, (n, r), generator=g).double()
        one[torch.rand(n, r, generator=g) < 0.5] = -1
        W = torch.zeros(n, features, r, dtype=torch.float64)
        v[:, 3], v[:, features - 2] = 1, m / 1024
        W[:, 3], W[:, features - 2] = one, one * k
        return v, W, one[ids], (one * k)[ids] * m[:, None] / 1024

    def along(p, Q):
        """p_i Q of the row's adapter"""
        out = torch.zeros(M, Q.shape[2], dtype=torch.float64)
        for a in range(n):
            out[ids == a] = p[ids == a] @ Q[a]
        return out

    def over_rows(p, q):
        return torch.stack([p[ids == a].t() @ q[ids == a] for a in range(n)])

    def same(got, want):
        assert float(want.abs().max()) <= 256 / 1024 and bool(want.any())
        assert torch.equal(got.double().cpu(), want)

    turns = torch.tensor([1.0, -1.0]).double().repeat(M // 2)[:, None]     # a row and the next: the same adapter, opposite values
    x, A, one, low = split(K)
    Bm, dy = whole(n, r, N), whole(M // 2, N).repeat_interleave(2, 0) * turns * (torch.rand(M // 2, 1, generator=g) < 100 / M).repeat_interleave(2, 0)
    out, saved = B.adapters_fwd(dev(x), dev(A), dev(Bm), ids.cuda(), base=dev(-along(one, Bm)))
    same(out, along(low, Bm))
    dB = B.adapters_bwd(dev(dy), dev(x), dev(A), dev(Bm), ids.cuda(), saved, need=(False, False, True))[2]
    same(dB, over_rows(low, dy))
    # and the other way: g in h's place
    dy, Bt, one, low = split(N)
    Bm, A, x = Bt.transpose(1, 2).contiguous(), whole(n, K, r), whole(M // 2, K).repeat_interleave(2, 0) * turns
    x *= (torch.rand(M // 2, 1, generator=g) < 100 / M).repeat_interleave(2, 0)
    At = A.transpose(1, 2).contiguous()
    _, saved = B.adapters_fwd(dev(x), dev(A), dev(Bm), ids.cuda())
    dx, dA, _ = B.adapters_bwd(dev(dy), dev(x), dev(A), dev(Bm), ids.cuda(), saved, base=dev(-along(one, At)), need=(True, True, False))
    same(dx, along(low, At))
    same(dA, over_rows(x, low))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M, K, N, r, n", [(9000, 72, 136, 32, 20), (1500, 70, 90, 12, 6), (6000, 100, 130, 8, 9), (250, 300, 260, 100, 2)])
def test_every_row_counts(M, K, N, r, n, dtype):
    """The gradients of A and B in whole numbers, exact: a row more or less in a sum is seen.  Sums stay under 256."""
    g = torch.Generator().manual_seed(M)
    whole = lambda share, *s: torch.randint(-1, 2, s, generator=g).double() * (torch.rand(s, generator=g) < share)
    x, dy, A, Bm = whole(0.5, M, K), whole(0.5, M, N), whole(1 / 16, n, K, r), whole(1 / 16, n, r, N)
    ids = torch.randint(-1, n, (M,), generator=g)
    want_A, want_B = torch.zeros(n, K, r, dtype=torch.float64), torch.zeros(n, r, N, dtype=torch.float64)
    for a in range(n):
        xa, ga = x[ids == a], dy[ids == a]
        want_A[a], want_B[a] = xa.t() @ (ga @ Bm[a].t()), (xa @ A[a]).t() @ ga
    assert 10 < float(want_A.abs().max()) <= 256 and 10 < float(want_B.abs().max()) <= 256
    dev = lambda t: t.to(dtype).cuda()
    _, saved = B.adapters_fwd(dev(x), dev(A), dev(Bm), ids.cuda())
    _, dA, dB = B.adapters_bwd(dev(dy), dev(x), dev(A), dev(Bm), ids.cuda(), saved)
    assert torch.equal(dA.double().cpu(), want_A) and torch.equal(dB.double().cpu(), want_B)
