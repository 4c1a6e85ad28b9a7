"""Dropout from the counter-based generator: which elements, and what becomes of them.

The mask is compared bit by bit.  Values: a product with the rate, itself rounded to 24 bits, and a sum, rounded once: 2^-24 (the rate)
and 2^-24 (the result) of the larger of the two terms in fp32; in bfloat16 the result's own 2^-8 / 2 = 2^-9 besides, of which a half
step of 8 bits is at most 2^-8 of the value."""
import pytest
import torch

from paper_2310_03675_amd import binding as B
from residual_block import bound, dropped, kept, rate

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def new(n, dtype, seed=0, shape=None):
    x = torch.randn(n, generator=torch.Generator().manual_seed(seed)).to(dtype)
    x[x == 0] = 1.0                                   # (a zero does not tell whether it was dropped)
    return (x if shape is None else x.reshape(shape)).cuda()


def near(got, want, terms, dtype):
    tol = 2.0 ** -22 * terms + (2.0 ** -8 * want.abs() if dtype == BF16 else 0)
    assert bool(((got.double().cpu() - want).abs() <= tol).all())


@pytest.mark.parametrize("n", [1, 7, 8, 9, 64, 2047, 2049, 100003, 1 << 20])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("p", [0.5, 0.1, 0.37, 0.999])
def test_against_the_definition(n, dtype, p):
    d = B.Dropout(p, seed=2 ** 63 + 12345, tensor_id=2 ** 32 - 3)
    x, r = new(n, dtype), new(n, dtype, 1)
    y = B.dropout(x, d)
    mask = kept(n, p, d.seed, d.tensor_id)
    assert torch.equal((y != 0).cpu(), mask)
    near(y, dropped(x, d), x.double().cpu().abs() * rate(p), dtype)
    z = B.dropout(x, d, residual=r)
    assert torch.equal(z.cpu()[~mask], r.cpu()[~mask])
    near(z, r.double().cpu() + dropped(x, d), x.double().cpu().abs() * rate(p) + r.double().cpu().abs(), dtype)
    # in place, either way
    for out in (x.clone(), r.clone()):
        a, b = (out, r) if torch.equal(out, x) else (x, out)
        assert B.dropout(a, d, residual=b, out=out) is out and torch.equal(out, z)
    v = x.clone()
    assert B.dropout(v, d, out=v) is v and torch.equal(v, y)


def test_the_lower_half_decides_at_the_bound():
    """Among four million elements some 60 have the bound's upper half; a bound just above and just below them differs there alone."""
    n, top = 1 << 22, 0x2345
    x = torch.ones(n, device="cuda")
    for low in (0, 1, 0x8000, 0xFFFF):
        p = (top * 65536 + low) / 2 ** 32
        assert bound(p) == top * 65536 + low
        assert torch.equal((B.dropout(x, B.Dropout(p, 5, 6)) != 0).cpu(), kept(n, p, 5, 6))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_all_and_none(dtype):
    x, r = new(1000, dtype), new(1000, dtype, 1)
    assert torch.equal(B.dropout(x, B.Dropout(0.0, 1, 2)), x)
    assert torch.equal(B.dropout(x, B.Dropout(2.0 ** -34, 1, 2)), x)
    assert not B.dropout(x, B.Dropout(1.0, 1, 2)).any()
    assert torch.equal(B.dropout(x, B.Dropout(1.0, 1, 2), residual=r), r)
    near(B.dropout(x, B.Dropout(0.0, 1, 2), residual=r), r.double().cpu() + x.double().cpu(), x.double().cpu().abs() + r.double().cpu().abs(), dtype)


def test_dropped_values_are_not_looked_at():
    d = B.Dropout(0.5, 3, 4)
    x, r = new(5000, F32), new(5000, F32, 1)
    mask = kept(5000, 0.5, 3, 4).cuda()
    bad = torch.where(mask, x, torch.where(torch.arange(5000, device="cuda") % 2 == 0, float("nan"), float("inf")))
    assert torch.equal(B.dropout(bad, d), B.dropout(x, d)) and torch.equal(B.dropout(bad, d, r), B.dropout(x, d, r))
    kept_bad = x.clone()
    kept_bad[mask] = float("inf")
    assert torch.equal(torch.isinf(B.dropout(kept_bad, d)), mask)


def test_streams_of_numbers():
    """Seeds, ids and steps are streams of their own; a share p of each is dropped, and of two a share p^2: within five deviations."""
    n, p = 1 << 20, 0.25
    x = torch.ones(n, device="cuda")
    masks = [B.dropout(x, d) != 0 for d in (B.Dropout(p, 1, 1), B.Dropout(p, 2, 1), B.Dropout(p, 1, 2), B.Dropout(p, 1 + 2 ** 32, 1),
                                            B.Dropout(p, 1, 1, torch.tensor(7, device="cuda")))]
    dev = lambda q: 5 * (q * (1 - q) * n) ** 0.5
    for i, m in enumerate(masks):
        assert abs(float((~m).sum()) - p * n) < dev(p)
        for o in masks[:i]:
            assert abs(float((~m & ~o).sum()) - p * p * n) < dev(p * p)
    assert torch.equal(masks[4], B.dropout(x, B.Dropout(p, 8, 1)) != 0)         # (seed + step)
    step = torch.tensor([-1], device="cuda")
    assert torch.equal(B.dropout(x, B.Dropout(p, 0, 1, step)), B.dropout(x, B.Dropout(p, 2 ** 64 - 1, 1)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off", [1, 3])
def test_tensors_that_start_anywhere(dtype, off):
    d = B.Dropout(0.3, 11, 12)
    whole = [new(4096 + off, dtype, k) for k in range(3)]
    x, r, out = (t[off:] for t in whole)
    want = B.dropout(x.clone(), d, residual=r.clone())
    head = whole[2][:off].clone()
    assert torch.equal(B.dropout(x, d, residual=r, out=out), want) and torch.equal(whole[2][:off], head)


def test_elements_beyond_32_bits():
    n = (1 << 31) + 1003
    x = torch.ones(n, dtype=BF16, device="cuda")
    d = B.Dropout(0.5, 21, 22)
    y = B.dropout(x, d, out=x)
    for first in (0, (1 << 31) - 500, n - 1001):
        assert torch.equal((y[first:first + 1000] != 0).cpu(), kept(1000, 0.5, 21, 22, first))
    assert torch.equal((y[-1:] != 0).cpu(), kept(1, 0.5, 21, 22, n - 1))


def test_graph_replays_take_the_step():
    """A captured call: every replay reads the step, and gives what an eager call gives."""
    x, step, out = new(100_001, F32), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty(100_001, device="cuda")
    d = B.Dropout(0.4, 31, 32, step)
    B.dropout(x, d, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dropout(x, d, out=out)
        step.add_(1)
    step.zero_()
    for k in range(4):
        x.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.dropout(x, B.Dropout(0.4, 31 + k, 32)))
        assert int(step) == k + 1


def test_side_stream():
    x, d = new(3_000_000, BF16), B.Dropout(0.2, 41, 42)
    want = B.dropout(x, d)
    late = torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late.copy_(x)
    got = B.dropout(late, d, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    torch.cuda.synchronize()
