"""Layer normalisation with the residual sum and the dropout in front of it, against 64 bits.

Tolerances, 2-norm of the difference over 2-norm of the result.  fp32: some ten roundings of 2^-24 between the inputs and y or ds, and
sums whose error is that of a few partial sums: 2e-6 (32 roundings).  bfloat16, of 8 significant bits: one rounding of at most 2^-8
more.  What is formed from the sum is compared with what the formulas make of the sum as it was held, the sum with its own.  ds is a
difference: against the 2-norm of its terms.  dweight and dbias: sums of terms of either sign, whose result may be smaller than its terms by the square root
of their number; against the 2-norm over the terms' own."""
import ctypes as C

import pytest
import torch

from paper_2310_03675_amd import binding as B
from residual_block import layer_norm

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def inputs(shape, dtype, seed=0, pdtype=F32, mean=0.5, std=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    C = shape[-1]
    x, res, dy, dsum = ((r(*shape) * std + mean).to(dtype).cuda() for _ in range(4))
    return x, res, dy, dsum, (1 + 0.3 * r(C)).to(pdtype).cuda(), (0.3 * r(C)).to(pdtype).cuda()


def near(got, want, tol, norm=None):
    d, n = (got.double().cpu().reshape(want.shape) - want).norm(), want.norm() if norm is None else norm
    assert d <= tol * n + 1e-30, (float(d), float(d / n) if n else None, tol)


def check(shape, dtype, how="plain", params="given", pdtype=F32, **k):
    """how: "plain", "residual", "dropout" or "both"."""
    x, res, dy, dsum, w, b = inputs(shape, dtype, pdtype=pdtype, **k)
    if params == "none":
        w = b = None
    d = B.Dropout(0.3, 77, 5) if how in ("dropout", "both") else None
    res, dsum = (res, dsum) if how in ("residual", "both") else (None, None)
    y, total, saved = B.layernorm_fwd(x, w, b, residual=res, dropout=d)
    want = layer_norm(x, dy, w, b, res, dsum, d, held=total)
    dx, dres, dw, db = B.layernorm_bwd(dy, total, saved, w, dsum, d)
    tol = 2e-6 + (2.0 ** -8 if dtype == BF16 else 0)
    near(total, want["sum"], tol)
    assert (total is x) == (how == "plain")
    near(y, want["y"], tol)
    near(dx, want["dx"], tol, norm=want["ds_terms"] / (0.7 if d is not None else 1.0))
    near(dres, want["dresidual"], tol, norm=want["ds_terms"])
    ptol = 0.0 if dw.dtype == F32 else 2.0 ** -8
    near(dw, want["dweight"], 1.0, norm=2e-6 * want["dw_terms"] + ptol * want["dweight"].norm())
    near(db, want["dbias"], 1.0, norm=2e-6 * want["db_terms"] + ptol * want["dbias"].norm())
    # what is not asked for changes nothing else
    only = B.layernorm_fwd(x, w, b, residual=res, dropout=d, need=(False, False))
    assert torch.equal(only[0], y) and only[2] is None and (only[1] is x or only[1] is None)
    for need in ((True, False, False, False), (False, True, False, False), (False, False, True, False), (False, False, False, True),
                 (True, True, False, False), (False, False, True, True)):
        got = B.layernorm_bwd(dy, total, saved, w, dsum, d, need=need)
        assert all((g is None) == (not n) and (g is None or torch.equal(g, v)) for g, n, v in zip(got, need, (dx, dres, dw, db)))
    # over their own inputs
    if res is not None:
        r2, x2 = res.clone(), x.clone()
        y2, t2, s2 = B.layernorm_fwd(x2, w, b, residual=r2, dropout=d, out=x2, out_sum=r2)
        assert y2 is x2 and t2 is r2 and torch.equal(y2, y) and torch.equal(t2, total) and torch.equal(s2, saved)
    else:
        x2 = x.clone()
        assert torch.equal(B.layernorm_fwd(x2, w, b, dropout=d, out=x2, need=(False, True))[0], y) and torch.equal(x2, y)


SHAPES = [(1, 1), (3, 1), (2, 2), (5, 7), (4, 8), (3, 9), (9, 12), (1, 561), (128, 512), (300, 24), (1000, 64), (33, 1031), (2, 3, 5, 40), (7, 4100),
          (5, 8192), (3, 16384), (3, 16385), (2, 30001), (2, 32768), (2, 32761), (20000, 8), (5000, 17), (3000, 130), (600, 2048), (2100, 4096)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", ["plain", "residual", "dropout", "both"])
def test_against_64_bits(shape, dtype, how):
    check(shape, dtype, how)


@pytest.mark.parametrize("shape", [(1000, 2051), (1000, 2048), (1023, 2056), (520, 4096), (1025, 2051), (2047, 1031), (2049, 1031)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_two_vectors(shape, dtype):
    """Two vectors to a thread, on both sides of how many rows take one launch, and of how many make parts."""
    check(shape, dtype, "both")


@pytest.mark.parametrize("how", ["plain", "both"])
def test_parameters(how):
    for dtype in (F32, BF16):
        check((50, 96), dtype, how, params="none")
        check((50, 99), dtype, how, params="none")
    check((50, 96), BF16, how, pdtype=BF16)
    check((50, 1031), BF16, how, pdtype=BF16)


def test_rows_of_one_value():
    """One column: nothing is left of it but the bias, and the gradient is none at all."""
    x, res, dy, dsum, w, b = inputs((100, 1), F32)
    y, s, saved = B.layernorm_fwd(x, w, b, residual=res)
    assert torch.equal(y, b.expand(100, 1))
    dx, dres, dw, _ = B.layernorm_bwd(dy, s, saved, w)
    assert not dx.any() and not dw.any()
    assert torch.equal(B.layernorm_bwd(dy, s, saved, w, dsum)[0], dsum)
    x = torch.full((4, 512), 3.25, device="cuda")
    y, _, saved = B.layernorm_fwd(x)
    assert not y.any() and torch.equal(saved[:, 0], torch.full((4,), 3.25, device="cuda"))


@pytest.mark.parametrize("C", [200, 5000])
def test_large_mean(C):
    """A mean that is many deviations away costs the bits it takes from x - mean, and no more."""
    x = (torch.randn(20, C, generator=torch.Generator().manual_seed(3)) + 1000.0).cuda()
    y, _, saved = B.layernorm_fwd(x)
    want = layer_norm(x, x)
    assert torch.allclose(saved[:, 0].double().cpu(), want["mean"], rtol=2.0 ** -22, atol=0)
    assert torch.allclose(saved[:, 1].double().cpu(), want["rstd"], rtol=1e-5, atol=0)
    assert float((y.double().cpu() - want["y"]).norm() / want["y"].norm()) < 1000 * 2.0 ** -23


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [24, 517, 9000])
def test_unusual_values_stay_in_their_row(dtype, C):
    x, res, dy, dsum, w, b = inputs((40, C), dtype)
    y0, s0, saved0 = B.layernorm_fwd(x, w, b, residual=res)
    dx0, _, _, db0 = B.layernorm_bwd(dy, s0, saved0, w, dsum)
    x[3, 5], x[17, C - 1], x[30, 0] = float("nan"), float("inf"), -float("inf")
    y, s, saved = B.layernorm_fwd(x, w, b, residual=res)
    dx, _, dw, db = B.layernorm_bwd(dy, s, saved, w, dsum)
    bad = torch.zeros(40, dtype=torch.bool)
    bad[[3, 17, 30]] = True
    assert bool(y[bad].isnan().all()) and bool(dx[bad].isnan().all()) and bool(dw.isnan().all())
    assert torch.equal(y[~bad], y0[~bad]) and torch.equal(dx[~bad], dx0[~bad]) and torch.equal(db, db0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [64, 513])
def test_tensors_that_start_anywhere(dtype, C):
    M, off = 70, 1
    flat = lambda t: torch.cat([t.new_zeros(off), t.reshape(-1)])[off:].reshape(t.shape)
    x, res, dy, dsum, w, b = inputs((M, C), dtype)
    d = B.Dropout(0.2, 1, 2)
    want = B.layernorm_fwd(x, w, b, residual=res, dropout=d)
    grads = B.layernorm_bwd(dy, want[1], want[2], w, dsum, d)
    ends = [torch.zeros(M * C + 2 * off, dtype=dtype, device="cuda") for _ in range(2)]
    out, total = (e[off:-off].reshape(M, C) for e in ends)
    got = B.layernorm_fwd(flat(x), flat(w), flat(b), residual=flat(res), dropout=d, out=out, out_sum=total)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and not any(e[0] or e[-1] for e in ends)
    assert all(torch.equal(p, q) for p, q in zip(B.layernorm_bwd(flat(dy), total, got[2], flat(w), flat(dsum), d), grads))


def test_rows_beyond_32_bits():
    C = 24
    M = (1 << 31) // C + 1000
    x = torch.empty(M, C, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    d = B.Dropout(0.5, 9, 10)
    y, s, saved = B.layernorm_fwd(x, dropout=d)
    dx = B.layernorm_bwd(x, s, saved, dropout=d, need=(True, False, False, False))[0]
    from residual_block import kept, rate
    for first in (0, (1 << 31) // C - 20, M - 40):
        rows = slice(first, first + 40)
        mask = kept(40 * C, 0.5, 9, 10, first * C).reshape(40, C)
        v = torch.where(mask, x[rows].double().cpu() * rate(0.5), torch.zeros((), dtype=torch.float64))
        assert torch.equal(s[rows].double().cpu(), v)          # (times two: exact)
        want = layer_norm(v.to(BF16), x[rows])
        near(y[rows], want["y"], 2e-6 + 2.0 ** -8)
        near(dx[rows], torch.where(mask, want["dresidual"] * 2, torch.zeros((), dtype=torch.float64)), 2e-6 + 2.0 ** -8, norm=2 * want["ds_terms"])


@pytest.mark.parametrize("M,C", [(3000, 512), (700, 4096), (100_000, 16)])
def test_same_bits_every_time(M, C):
    x, res, dy, dsum, w, b = inputs((M, C), BF16)
    d = B.Dropout(0.1, 1, 2)
    run = lambda: (lambda y, s, k: (y, s, k) + B.layernorm_bwd(dy, s, k, w, dsum, d))(*B.layernorm_fwd(x, w, b, residual=res, dropout=d))
    first = run()
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(run(), first))


def test_graph_and_side_stream():
    x, res, dy, dsum, w, b = inputs((1000, 520), F32)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = B.Dropout(0.3, 50, 3, step)

    def run():
        y, s, k = B.layernorm_fwd(x, w, b, residual=res, dropout=d)
        return (y, s, k) + B.layernorm_bwd(dy, s, k, w, dsum, d)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
        step.add_(1)
    step.zero_()
    for k in range(4):
        res.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        held, step_ = [t.clone() for t in got], int(step)
        assert step_ == k + 1
        step.fill_(k)
        assert all(torch.equal(p, q) for p, q in zip(held, run()))
        step.fill_(k + 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = torch.zeros_like(x)
        late.copy_(x)
    y, s, k = B.layernorm_fwd(late, w, b, residual=res, dropout=d, stream=side)
    grads = B.layernorm_bwd(dy, s, k, w, dsum, d, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip((y, s, k) + grads, run()))
    torch.cuda.synchronize()


def test_gradients_against_differences():
    """A directional derivative of a scalar of y and the sum, by central differences of the 64-bit formula, at the library's gradients."""
    x, res, dy, dsum, w, b = inputs((6, 40), F32)
    d = B.Dropout(0.25, 3, 4)
    y, s, saved = B.layernorm_fwd(x, w, b, residual=res, dropout=d)
    grads = dict(zip(("x", "res", "w"), B.layernorm_bwd(dy, s, saved, w, dsum, d)))
    at = {"x": x.double().cpu(), "res": res.double().cpu(), "w": w.double().cpu()}

    def value(v):
        r = layer_norm(v["x"], dy, v["w"], b, v["res"], dsum, d)
        return float((r["y"] * dy.double().cpu()).sum() + (r["sum"] * dsum.double().cpu()).sum())

    g = torch.Generator().manual_seed(8)
    for name, grad in grads.items():
        u = torch.randn(at[name].shape, generator=g, dtype=torch.float64)
        h = 1e-5
        step = lambda t: {**at, name: at[name] + t * u}
        want = (value(step(h)) - value(step(-h))) / (2 * h)
        assert abs(want - float((grad.double().cpu() * u).sum())) <= 1e-4 * float(grad.double().norm()) * float(u.norm()) / 10


@pytest.mark.parametrize("M", [1, 128, 300, 1024, 1025])
def test_gradients_over_their_own_inputs(M):
    """dx over dy and dresidual over dsum, as the interface allows: of few rows too, whose columns' sums read dy beside them."""
    x, res, dy, dsum, w, b = inputs((M, 512), F32)
    d = B.Dropout(0.3, 77, 5)
    _, total, saved = B.layernorm_fwd(x, w, b, residual=res, dropout=d)
    want = B.layernorm_bwd(dy, total, saved, w, dsum, d)
    first, apart = dy.clone(), [torch.empty_like(w), torch.empty_like(w)]
    lib = B.load()
    ws = torch.empty(lib.hdqt_layernorm_bwd_workspace_size(M, 512, 0), dtype=torch.uint8, device="cuda")
    p = lambda t: C.c_void_p(t.data_ptr())
    rc = lib.hdqt_layernorm_bwd(p(dy), p(dsum), p(total), C.byref(d.c()), p(w), p(saved), p(dy), p(dsum), p(apart[0]), p(apart[1]), M, 512, 0, 0,
                                p(ws), ws.numel(), C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    assert torch.equal(dy, want[0]) and torch.equal(dsum, want[1])
    exact = layer_norm(x, first, w, b, res, None, d, held=total)
    for got, name, terms in zip(apart, ("dweight", "dbias"), ("dw_terms", "db_terms")):
        near(got, exact[name], 1.0, norm=2e-6 * exact[terms])
