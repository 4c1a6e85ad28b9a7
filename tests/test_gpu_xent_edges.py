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


# ---- values that are not ordinary, at sizes that the large kernels multiply ----
#
# (rows, features, classes): small tiles, large ones, several pieces of the classes (of which fp32 alone makes dz from logits that
# a step has kept, where they are one)
LARGE = {F32: [(300, 264, 10007), (2600, 520, 8003), (9001, 72, 6001)],
         BF16: [(300, 264, 6200), (4100, 2056, 12011), (203, 40, 70001)]}
EACH = [(dtype, *size) for dtype in LARGE for size in LARGE[dtype]]
each_large = pytest.mark.parametrize("dtype,M,K,N", EACH, ids=lambda v: str(v).replace("torch.", ""))


def inputs(M, K, N, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return (r(M, K).to(dtype), (r(K, N) * 1.5 / math.sqrt(K)).to(dtype), (r(N) * 0.5).to(dtype),
            torch.randint(0, N, (M,), generator=g, device="cuda"))


def reference(X, W, b, t, ignore=IGNORE):
    """Loss, dX, dW, db of the mean in 64 bits, and the 2-norm of dz."""
    X, W = X.double(), W.double()
    z = X @ W + b.double()
    lse = torch.logsumexp(z, 1)
    keep = t != ignore
    at = torch.where(keep, t, torch.zeros_like(t))[:, None]
    share = 1.0 / max(1, int(keep.sum()))
    loss = torch.where(keep, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse)).sum() * share
    dz = torch.exp(z - lse[:, None]).scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None]) * (keep.double() * share)[:, None]
    return loss, dz @ W.t().contiguous(), X.t().contiguous() @ dz, dz.sum(0), float(dz.norm())


def tolerance(dtype, K):
    return (1e-5 if K <= 1000 else 4e-5) if dtype == F32 else 2.0 ** -7 + 4e-5


def both_ways(X, W, t, b, **how):
    """A step's results, which are those of the two calls apart."""
    step = B.xent_step(X, W, t, b, **how)
    loss, saved = B.xent_fwd(X, W, t, b, **how)
    apart = (loss,) + tuple(B.xent_bwd(None, X, W, t, saved, b, **how))
    for p, q in zip(step, apart):
        assert torch.equal(p.isnan(), q.isnan()) and torch.equal(p.nan_to_num(), q.nan_to_num())
    return step


@each_large
def test_no_row_counts(dtype, M, K, N):
    X, W, b, t = inputs(M, K, N, dtype)
    t.fill_(IGNORE)
    for reduction in ("mean", "sum", "none"):
        for v in both_ways(X, W, t, b, reduction=reduction):
            assert not v.any()
    t[M // 2] = N - 1
    loss, dX, dW, db = both_ways(X, W, t, b)
    want = reference(X, W, b, t)
    near(loss, want[0], 4e-5)
    near(dX, want[1], tolerance(dtype, K))
    near(dW, want[2], tolerance(dtype, K), want[4])
    near(db, want[3], tolerance(dtype, K), want[4])
    assert not dX[:M // 2].any() and not dX[M // 2 + 1:].any()
    # another number to ignore, a class among them
    loss, dX, _, _ = B.xent_step(X, W, t, b, ignore_index=N - 1)
    assert not dX[M // 2].any() and bool(loss.isnan())          # (-100 is no class then)


@each_large
def test_classes_taken_out(dtype, M, K, N):
    """Minus infinity, and half the type's lowest value, as a class's bias: no probability, no gradient."""
    X, W, b, t = inputs(M, K, N, dtype)
    half = N // 2
    t = t % half
    want = reference(X, W[:, :half], b[:half], t)
    for lowest in (-math.inf, torch.finfo(dtype).min / 2):
        v = b.clone()
        v[half:] = lowest
        loss, dX, dW, db = both_ways(X, W, t, v)
        near(loss, want[0], 4e-5)
        near(dX, want[1], tolerance(dtype, K))
        near(dW[:, :half], want[2], tolerance(dtype, K), want[4])
        near(db[:half], want[3], tolerance(dtype, K), want[4])
        assert not dW[:, half:].any() and not db[half:].any()
    # a target that is taken out: the loss is infinite, the gradient that of the others' probabilities
    v = b.clone()
    v[half:] = -math.inf
    t2 = t.clone()
    t2[5] = N - 1
    loss, dX, dW, db = both_ways(X, W, t2, v, reduction="none")
    assert float(loss[5]) == math.inf and bool(loss[:5].isfinite().all()) and bool(loss[6:].isfinite().all())
    assert bool(dX.isfinite().all()) and bool(dW.isfinite().all()) and float(db[N - 1]) == -1.0
    # every class
    loss, dX, dW, db = both_ways(X, W, t, torch.full_like(b, -math.inf), reduction="none")
    assert bool((loss == math.inf).all()) and bool(dX.isfinite().all()) and bool(dW.isfinite().all())


@each_large
def test_values_that_are_not_finite_stay_in_their_row(dtype, M, K, N):
    X, W, b, t = inputs(M, K, N, dtype)
    clean, dX0, dW0, _ = B.xent_step(X, W, t, b, reduction="none")
    rest, at = torch.ones(M, dtype=torch.bool, device="cuda"), M - 2
    rest[at] = False
    X2 = X.clone()
    X2[at, 3] = math.nan
    loss, dX, dW, db = both_ways(X2, W, t, b, reduction="none")
    assert bool(loss[at].isnan()) and torch.equal(loss[rest], clean[rest])
    assert bool(dX[at].isnan().all()) and torch.equal(dX[rest], dX0[rest])
    assert bool(dW.isnan().all()) and bool(db.isnan().all())    # (sums over all rows)
    v = b.clone()
    v[N - 3] = math.inf
    loss, dX, _, _ = both_ways(X, W, t, v, reduction="none")
    assert bool(loss.isnan().all()) and bool(dX.isnan().all())
    for bad in (N, -1, 1 << 40, -(1 << 40)):                    # no classes
        t2 = t.clone()
        t2[at] = bad
        loss, dX, _, _ = both_ways(X, W, t2, b, reduction="none")
        assert bool(loss[at].isnan()) and bool(dX[at].isnan().all())
        assert torch.equal(loss[rest], clean[rest]) and torch.equal(dX[rest], dX0[rest])
        # a row that is ignored may hold anything
        loss, dX, dW, _ = both_ways(X, W, t2, b, reduction="none", ignore_index=bad)
        assert float(loss[at]) == 0.0 and not dX[at].any() and bool(dW.isfinite().all())
    # and its features too, but for the gradient of the weight, in which zero times NaN is none
    loss, dX, _, db = both_ways(X2, W, t2, b, reduction="none", ignore_index=bad)
    assert float(loss[at]) == 0.0 and not dX[at].any() and bool(db.isfinite().all()) and torch.equal(dX[rest], dX0[rest])


@each_large
def test_large_logits(dtype, M, K, N):
    """Logits of +-3e4: exponentials only relative to the largest.  Logits of +-1e-26: all classes alike."""
    X, W, b, t = inputs(M, K, N, dtype)
    X = X * 8192
    loss, dX, dW, _ = both_ways(X, W, t, b)
    near(loss, reference(X, W, b, t)[0], 4e-5)
    assert bool(dX.isfinite().all()) and bool(dW.isfinite().all())
    tiny, none = (X * 1e-30).contiguous(), torch.zeros_like(b)
    loss, dX, _, db = both_ways(tiny, W, t, none)
    want = reference(tiny, W, none, t)
    near(loss, want[0], 4e-5)
    near(dX, want[1], tolerance(dtype, K))
    near(db, want[3], tolerance(dtype, K), want[4])


@pytest.mark.parametrize("M,K,N", LARGE[F32])
def test_gradient_by_differences(M, K, N):
    """The sum of the losses along a direction that moves logits by about one, against (f(x + h d) - f(x - h d)) / 2h with
    h = 1/128, rows' losses added up in 64 bits.  The derivative is of the size of sqrt(M).  A row's third derivative, of
    either sign, is at most about 4: sqrt(M) 4 h^2 / 6, 4e-5 sqrt(M); a row's loss of 10 is off by 10 sqrt(K) 2^-24, 1.4e-5,
    over 2 h: 1e-3 sqrt(M).  Twice that."""
    X, W, b, t = inputs(M, K, N, F32)
    t[::7] = IGNORE
    _, dX, dW, db = B.xent_step(X, W, t, b, reduction="sum")
    f = lambda X, W, b: float(B.xent_fwd(X, W, t, b, reduction="none")[0].double().sum())
    g, h = torch.Generator(device="cuda").manual_seed(3), 1 / 128
    d, e, c = (torch.randn(v.shape, generator=g, device="cuda") for v in (X, W, b))
    e /= math.sqrt(K)
    for got, plus, minus in ((dX.double() * d, (X + h * d, W, b), (X - h * d, W, b)), (dW.double() * e, (X, W + h * e, b), (X, W - h * e, b)),
                             (db.double() * c, (X, W, b + h * c), (X, W, b - h * c))):
        assert float(got.sum()) == pytest.approx((f(*plus) - f(*minus)) / (2 * h), rel=0, abs=2e-3 * math.sqrt(M))
