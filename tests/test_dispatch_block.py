"""What a residual block's operators launch, at the edges of their rules and of what they take (host code: nothing is launched)."""
import math
import random

import pytest

from dispatch_block import dispatch

F32, BF16 = 0, 1
ROWS, FEATURES = 65535 * 64, 1 << 21


def test_the_largest_that_are_taken_are_launched():
    calls = [("dropout", 1 << 40, t) for t in (F32, BF16)]
    for M, C in (((1 << 31) - 1, 1), ((1 << 31) - 1, 32768), (1, 32768), ((1 << 31) - 1, 65), (1 << 20, 8193)):
        for t in (F32, BF16):
            calls += [("norm_fwd", M, C, t), ("norm_bwd", M, C, t, 15)]
    for M, K, N, r, n in ((ROWS, 1, 1, 1, 1), (ROWS, 70, 80, 128, 1024), (1, FEATURES, FEATURES, 128, 1), (300, FEATURES, FEATURES, 1, 1024),
                          (ROWS, 4096, FEATURES, 16, 1024), (1, FEATURES, 1, 3, 1024), (257, 1, FEATURES, 17, 1024)):
        for t in (F32, BF16):
            calls += [("adapt_fwd", M, K, N, r, n, t), ("adapt_bwd", M, K, N, r, n, t, 7)]
    for what, call in zip(calls, dispatch(calls)):
        assert call.rc == 0 and call.launches, (what, call)


def test_launches():
    """A plan for more rows than a wave sees at once; both ways in one launch where a tile is small; sums of parts where workgroups are few."""
    names = lambda *c: [k.replace("_kernel", "") for k in dispatch([c])[0].kernels]
    assert names("dropout", 1000, F32) == ["dropout"]
    assert names("norm_fwd", 1000, 64, F32) == ["layernorm_fwd"]
    assert names("norm_bwd", 1025, 64, F32, 15) == ["layernorm_bwd", "layernorm_params"]
    assert names("norm_bwd", 1025, 64, F32, 3) == ["layernorm_bwd"] and names("norm_bwd", 1024, 64, F32, 15) == ["layernorm_bwd"]
    # (over dy only behind whoever else reads it)
    assert names("norm_bwd", 1024, 64, F32, 15 + 16) == ["layernorm_bwd", "layernorm_params"] == names("norm_bwd", 1024, 64, F32, 15 + 32)
    assert names("adapt_fwd", 100, 256, 256, 8, 4, F32) == ["down_up"]
    assert names("adapt_fwd", 257, 256, 256, 8, 4, F32) == ["plan", "down_up"]
    assert names("adapt_fwd", 256, 256, 256, 8, 4, F32) == ["down_up"] and names("adapt_fwd", 128, 4096, 4096, 16, 4, BF16) == ["down", "up"]
    assert names("adapt_fwd", 129, 4096, 4096, 16, 4, BF16) == ["plan", "down", "up"]
    assert names("adapt_fwd", 8192, 256, 256, 8, 4, F32)[0] == "plan"
    assert names("adapt_fwd", 8193, 256, 256, 8, 4, F32) == ["plan_count", "plan_starts", "plan_order", "down", "up"]
    assert names("adapt_fwd", 100, 256, 63, 8, 4, F32) == ["down", "up"] and names("adapt_fwd", 100, 31, 256, 8, 4, F32) == ["down", "up"]
    assert names("adapt_fwd", 100, 256, 256, 65, 4, F32) == ["down", "up"] and names("adapt_fwd", 5000, 256, 256, 8, 4, F32) == ["plan", "down", "up"]
    assert names("adapt_fwd", 100, 4096, 4096, 8, 4, F32) == ["down", "up"]
    assert names("adapt_bwd", 100, 256, 256, 8, 4, F32, 7) == ["down_up", "weights"]
    assert names("adapt_bwd", 100, 256, 256, 8, 4, F32, 6) == ["down", "weights"] and names("adapt_bwd", 100, 256, 256, 8, 4, F32, 4) == ["weights"]
    assert names("adapt_bwd", 100, 256, 256, 4, 4, BF16, 1) == ["down", "up"]
    assert names("adapt_bwd", 8192, 512, 512, 8, 2, F32, 7) == ["down", "up", "weights", "add_parts"]


def _size(rng, lo, hi):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return rng.choice((lo, hi, max(lo, min(hi, round(v))), max(lo, min(hi, round(v))), max(lo, min(hi, round(v)))))


@pytest.mark.parametrize("seed", range(4))
def test_whatever_is_taken_is_launched(seed):
    rng = random.Random(seed)
    calls = []
    for _ in range(400):
        t = rng.choice((F32, BF16))
        M, C = _size(rng, 1, (1 << 31) - 1), _size(rng, 1, 32768)
        calls += [("dropout", _size(rng, 1, 1 << 40), t), ("norm_fwd", M, C, t), ("norm_bwd", M, C, t, rng.randint(1, 15))]
        size = _size(rng, 1, ROWS), _size(rng, 1, FEATURES), _size(rng, 1, FEATURES), _size(rng, 1, 128), _size(rng, 1, 1024), t
        calls += [("adapt_fwd", *size), ("adapt_bwd", *size, rng.randint(1, 7))]
    for what, call in zip(calls, dispatch(calls)):
        assert call.rc == 0, (what, call)
