"""Low-rank adapters of many rows beside a shared projection, against 64 bits.

Tolerances, 2-norm of the difference over the 2-norm of the result or, where terms cancel, of what it is a sum of.  fp32: two products
one after the other, each with sums in 32 bits over several waves' parts: 2e-6 (32 roundings of 2^-24) of the terms.
bfloat16: the sums the same, h and g in the second product off by 2^-16 of themselves (1.6e-5), one rounding of the result of at most
2^-8."""
import pytest
import torch

from paper_2310_03675_amd import binding as B
from residual_block import adapters

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def inputs(M, K, N, r, n, dtype, seed=0, none=0.2, scale=True):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dtype).cuda()
    ids = torch.randint(0, n, (M,), generator=g)
    ids[torch.rand(M, generator=g) < none] = -1
    return dict(x=f(M, K), A=f(n, K, r, std=K ** -0.5), Bm=f(n, r, N, std=r ** -0.5), ids=ids.cuda(),
                scale=(torch.rand(n, generator=g) + 0.5).cuda() if scale else None, base=f(M, N), dy=f(M, N), dbase=f(M, K))


def near(got, want, dtype, norm=None):
    tol = 2e-6 if dtype == F32 else 2e-6 + 1.6e-5 + 2.0 ** -8
    d, n = float((got.double().cpu() - want).norm()), float(want.norm()) if norm is None else norm
    assert got.shape == want.shape and d <= tol * n + 1e-30, (d, d / n if n else None, tol)


def terms(i):
    """Sizes of what out and dx, dA and dB are sums of: the base, and a bound of the products by their factors."""
    K, r, N = i["A"].shape[1], i["A"].shape[2], i["Bm"].shape[2]
    x, dy, A, Bm = (i[k].double() for k in ("x", "dy", "A", "Bm"))
    a, b = float(A.abs().max()), float(Bm.abs().max())
    # |x| |A| |B| by rows: no more than the rows' norms times the factors' largest, and the square root of what is summed
    return (float(i["base"].double().norm()) + 1.5 * float(x.norm()) * a * b * (r * N) ** 0.5,
            float(i["dbase"].double().norm()) + 1.5 * float(dy.norm()) * a * b * (r * K) ** 0.5)


def check(M, K, N, r, n, dtype, **k):
    i = inputs(M, K, N, r, n, dtype, **k)
    want = adapters(*(i[q] for q in ("x", "A", "Bm", "ids", "scale", "base", "dy", "dbase")))
    copies = {q: t.clone() for q, t in i.items() if t is not None}
    out, saved = B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"], i["base"])
    dx, dA, dB = B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"], base=i["dbase"])
    assert all(torch.equal(i[q], t) for q, t in copies.items())
    t_out, t_dx = terms(i)
    near(out, want["out"], dtype, norm=min(float(want["out"].norm()) * 4, t_out))
    near(dx, want["dx"], dtype, norm=min(float(want["dx"].norm()) * 4, t_dx))
    near(dA, want["dA"], dtype, norm=4 * float(want["dA"].norm()))
    near(dB, want["dB"], dtype, norm=4 * float(want["dB"].norm()))
    # rows without an adapter are the base's, adapters without a row have no gradient
    none = i["ids"] < 0
    assert torch.equal(out[none], i["base"][none]) and torch.equal(dx[none], i["dbase"][none])
    idle = [a for a in range(n) if not bool((i["ids"] == a).any())]
    assert not dA[idle].any() and not dB[idle].any()
    # without a base, and over it
    bare, _ = B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"])
    assert not bare[none].any()
    near(bare, adapters(i["x"], i["A"], i["Bm"], i["ids"], i["scale"])["out"], dtype, norm=t_out)
    over = i["base"].clone()
    assert B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"], over, out=over)[0] is over and torch.equal(over, out)
    over = i["dbase"].clone()
    assert B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"], base=over, out=over)[0] is over and torch.equal(over, dx)
    # what is not asked for changes nothing else
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        got = B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"], base=i["dbase"], need=need)
        assert all((q is None) == (not w) and (q is None or torch.equal(q, v)) for q, w, v in zip(got, need, (dx, dA, dB)))


SIZES = [(1, 1, 1, 1, 1), (1, 561, 512, 8, 10), (2, 64, 128, 16, 3), (3, 7, 5, 2, 2), (17, 33, 31, 3, 4), (32, 63, 127, 4, 5), (33, 65, 129, 5, 1),
         (64, 512, 640, 16, 40), (64, 100, 100, 17, 2), (65, 100, 100, 33, 3), (65, 96, 1, 1, 1), (70, 1, 70, 64, 2), (100, 40, 300, 24, 7),
         (128, 512, 512, 8, 10), (200, 1153, 331, 31, 6), (257, 300, 1000, 128, 3), (300, 1031, 259, 100, 5), (500, 24, 24, 65, 300),
         (1000, 320, 70, 7, 1000), (1500, 200, 333, 12, 1), (4000, 130, 60, 16, 2), (9000, 72, 136, 32, 20)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_against_64_bits(size, dtype):
    check(*size, dtype)


@pytest.mark.parametrize("r", [1, 2, 3, 4, 6, 8, 9, 16, 20, 32, 34, 48, 64, 66, 96, 127, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ranks(r, dtype):
    check(90, 200, 264, r, 3, dtype, seed=r)
    check(20, 130, 129, r, 3, dtype, seed=r, scale=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [31, 32, 33, 63, 64, 65, 96, 97, 128, 129, 255, 256, 257, 1023, 1025])
def test_rows_around_tiles(M, dtype):
    check(M, 80, 140, 8, 1, dtype, none=0.0)
    check(M, 80, 140, 8, 2, dtype, none=0.9)
    check(M, 80, 140, 8, 2, dtype, none=1.0)


@pytest.mark.parametrize("M, n", [(8191, 3), (8192, 1024), (8193, 3), (16385, 1), (24577, 1024), (70001, 10)])
def test_plans_of_many_rows(M, n):
    """On both sides of what one workgroup of the plan looks through, rows without an adapter and with a wrong one among them."""
    i = inputs(M, 40, 72, 4, n, BF16)
    i["ids"][M // 2], i["ids"][M - 1] = n, n - 1
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    bad[M // 2] = True
    out, saved = B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"], i["base"])
    dx, dA, dB = B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"])
    want = adapters(i["x"], i["A"], i["Bm"], torch.where(bad, torch.full_like(i["ids"], -1), i["ids"]), i["scale"], i["base"], i["dy"])
    assert bool(out[bad].isnan().all()) and bool(dx[bad].isnan().all())
    good = ~bad.cpu()
    near(out[~bad], want["out"][good], BF16)
    near(dx[~bad], want["dx"][good], BF16)
    near(dA, want["dA"], BF16)
    near(dB, want["dB"], BF16)


@pytest.mark.parametrize("M", [50, 150, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_numbers_that_are_none(M, dtype):
    """At n or above: the row is NaN, and nothing is read or added for it."""
    i = inputs(M, 96, 200, 8, 4, dtype)
    ids = i["ids"].clone()
    ids[3], ids[M - 1], ids[7] = 4, 2 ** 62, -2 ** 62
    out, saved = B.adapters_fwd(i["x"], i["A"], i["Bm"], ids, i["scale"], i["base"])
    dx, dA, dB = B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], ids, saved, i["scale"])
    bad = torch.zeros(M, dtype=torch.bool)
    bad[[3, M - 1]] = True
    assert torch.equal(out.isnan().all(1).cpu(), bad) and torch.equal(dx.isnan().all(1).cpu(), bad)
    assert torch.equal(out.isnan().any(1).cpu(), bad) and torch.equal(out[7], i["base"][7])
    masked = torch.where(bad.cuda(), torch.full_like(ids, -1), ids)
    want = adapters(i["x"], i["A"], i["Bm"], masked, i["scale"], None, i["dy"])
    near(dA, want["dA"], dtype)
    near(dB, want["dB"], dtype)


@pytest.mark.parametrize("M", [40, 300])
def test_an_adapter_without_rows(M):
    """Zeros for its gradients, whatever its matrices and its scale hold; the others as without it."""
    i = inputs(M, 96, 200, 8, 4, F32)
    ids = torch.where(i["ids"] == 2, torch.full_like(i["ids"], 1), i["ids"])
    run = lambda: (B.adapters_fwd(i["x"], i["A"], i["Bm"], ids, i["scale"], i["base"]))
    out, saved = run()
    grads = B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], ids, saved, i["scale"])
    i["scale"][2], i["A"][2], i["Bm"][2] = float("inf"), float("nan"), float("inf")
    out2, saved = run()
    got = B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], ids, saved, i["scale"])
    assert torch.equal(out2, out) and all(torch.equal(p, q) for p, q in zip(got, grads))
    assert not got[1][2].any() and not got[2][2].any()


@pytest.mark.parametrize("M", [40, 200, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_unusual_values_stay_where_they_belong(M, dtype):
    """A row's NaN is that row's out, and its adapter's gradients; an infinity gives infinities or NaN; other rows have the same bits."""
    i = inputs(M, 130, 140, 12, 5, dtype, none=0.0)
    run = lambda: B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"], i["base"])
    bwd = lambda saved: B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"])
    out0, saved = run()
    dx0, dA0, dB0 = bwd(saved)
    i["x"][9, 129], i["x"][20, 0], i["dy"][30, 5] = float("nan"), float("inf"), float("nan")
    out, saved = run()
    dx, dA, dB = bwd(saved)
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    bad[[9, 20]] = True
    assert bool(out[9].isnan().all()) and not out[20].isfinite().any() and torch.equal(out[~bad], out0[~bad])
    dbad = torch.zeros(M, dtype=torch.bool, device="cuda")
    dbad[30] = True
    assert bool(dx[30].isnan().all()) and torch.equal(dx[~dbad], dx0[~dbad])
    a9, a20, a30 = (int(i["ids"][k]) for k in (9, 20, 30))
    touched = {a9, a20, a30}
    assert bool(dB[a9].isnan().all()) and bool(dA[a9][129].isnan().all()) and bool(dA[a30].isnan().all())
    for a in set(range(5)) - touched:
        assert torch.equal(dA[a], dA0[a]) and torch.equal(dB[a], dB0[a])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(30, 100, 136, 8, 3), (90, 101, 135, 20, 3)], ids=str)
def test_tensors_that_start_anywhere(dtype, size):
    i = inputs(*size, dtype)
    flat = lambda t: None if t is None else torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].reshape(t.shape)
    f = {k: t if k in ("ids", "scale") else flat(t) for k, t in i.items()}
    out, saved = B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"], i["base"])
    grads = B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"], base=i["dbase"])
    M, N = out.shape
    ends = torch.zeros(M * N + 2, dtype=dtype, device="cuda")
    got, saved = B.adapters_fwd(f["x"], f["A"], f["Bm"], f["ids"], f["scale"], f["base"], out=ends[1:-1].reshape(M, N))
    assert torch.equal(got, out) and not ends[0] and not ends[-1]
    assert all(torch.equal(p, q) for p, q in zip(grads, B.adapters_bwd(f["dy"], f["x"], f["A"], f["Bm"], f["ids"], saved, f["scale"], base=f["dbase"])))


def test_rows_beyond_32_bits():
    """2.2 G elements of x and of out: the last rows are read and written."""
    M, K, N, r, n = 34000, 65536, 65600, 4, 2
    g = torch.Generator(device="cuda").manual_seed(0)
    new = lambda *s: torch.empty(*s, dtype=BF16, device="cuda").normal_(generator=g)
    x, A, Bm, ids = new(M, K), new(n, K, r) * K ** -0.5, new(n, r, N), torch.randint(0, n, (M,), device="cuda", generator=g)
    out, saved = B.adapters_fwd(x, A, Bm, ids)
    for first in (0, (1 << 31) // N - 5, M - 10):
        rows = slice(first, first + 10)
        near(out[rows], adapters(x[rows], A, Bm, ids[rows])["out"], BF16)
    dx = B.adapters_bwd(out, x, A, Bm, ids, saved, need=(True, False, False), out=x)[0]
    for first in (0, M - 10):
        rows = slice(first, first + 10)
        near(dx[rows], adapters(out[rows][:, :K] * 0, A, Bm, ids[rows], dy=out[rows])["dx"], BF16)


@pytest.mark.parametrize("size", [(50, 700, 600, 8, 9), (4000, 512, 384, 16, 12)], ids=str)
def test_same_bits_every_time(size):
    i = inputs(*size, BF16)

    def run():
        out, saved = B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"], i["base"])
        return (out,) + B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"])

    first = run()
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(run(), first))


@pytest.mark.parametrize("size", [(40, 300, 256, 8, 5), (700, 256, 300, 16, 6)], ids=str)
def test_graph_and_side_stream(size):
    """Captured with one assignment of rows to adapters, replayed with others."""
    i = inputs(*size, F32)
    ids = i["ids"]

    def run(**k):
        out, saved = B.adapters_fwd(i["x"], i["A"], i["Bm"], ids, i["scale"], i["base"], **k)
        return (out,) + B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], ids, saved, i["scale"], **k)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for k in range(4):
        ids.copy_((ids + 2 + k) % (size[4] + 1) - 1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, run()))
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    torch.cuda.synchronize()


def test_gradients_against_differences():
    i = inputs(20, 30, 40, 6, 3, F32)
    _, saved = B.adapters_fwd(i["x"], i["A"], i["Bm"], i["ids"], i["scale"], i["base"])
    grads = dict(zip(("x", "A", "Bm"), B.adapters_bwd(i["dy"], i["x"], i["A"], i["Bm"], i["ids"], saved, i["scale"])))
    at = {k: i[k].double().cpu() for k in ("x", "A", "Bm")}
    value = lambda v: float((adapters(v["x"], v["A"], v["Bm"], i["ids"], i["scale"])["out"] * i["dy"].double().cpu()).sum())
    g = torch.Generator().manual_seed(8)
    for name, grad in grads.items():
        u = torch.randn(at[name].shape, generator=g, dtype=torch.float64)
        want = (value({**at, name: at[name] + 1e-3 * u}) - value({**at, name: at[name] - 1e-3 * u})) / 2e-3      # (linear in each: exact)
        assert abs(want - float((grad.double().cpu() * u).sum())) <= 1e-5 * float(grad.double().norm()) * float(u.norm())
