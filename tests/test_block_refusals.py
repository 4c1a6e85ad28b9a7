"""Calls of a residual block's operators that are refused: on the host, before anything is launched (no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2310_03675_amd import autograd as A
from paper_2310_03675_amd import binding as B

FAKE = C.c_void_p(0x10000)
ODD = C.c_void_p(0x10001)
NULL, DIM, WORKSPACE, ALIGN, DTYPE, OPTION = -1, -2, -10, -11, -15, -16


def _with(ok, **changes):
    return tuple({**ok, **changes}.values())


def _drop(p=0.5, step=None):
    return C.byref(B.CDropout(p, 1, step, 2, 0))


def test_dropout_refusals():
    lib = B.load()
    call = lambda **k: lib.hdqt_dropout(*_with(dict(x=FAKE, residual=FAKE, y=FAKE, n=100, dtype=0, d=_drop(), stream=None), **k))
    for what in ("x", "y", "d"):
        assert call(**{what: None}) == NULL, what
    assert call(n=0) == DIM and call(n=-1) == DIM and call(n=(1 << 40) + 1) == DIM
    assert call(dtype=2) == DTYPE
    for what in ("x", "residual", "y"):
        assert call(**{what: ODD}) == ALIGN, what
    for p in (-0.1, 1.1, float("nan"), float("inf")):
        assert call(d=_drop(p)) == OPTION, p
    assert call(d=_drop(step=0x10004)) == ALIGN


def _norm(name, **changes):
    lib = B.load()
    if name == "fwd":
        return lib.hdqt_layernorm_fwd(*_with(dict(x=FAKE, residual=FAKE, dropout=_drop(), weight=FAKE, bias=FAKE, sum=FAKE, y=FAKE, saved=FAKE,
                                                  M=10, C=64, eps=1e-5, dtype=0, pdtype=0, stream=None), **changes))
    return lib.hdqt_layernorm_bwd(*_with(dict(dy=FAKE, dsum=FAKE, s=FAKE, dropout=_drop(), weight=FAKE, saved=FAKE, dx=FAKE, dresidual=FAKE,
                                              dweight=FAKE, dbias=FAKE, M=10, C=64, dtype=0, pdtype=0, ws=FAKE, bytes=1 << 30, stream=None),
                                         **changes))


@pytest.mark.parametrize("name", ["fwd", "bwd"])
def test_layernorm_refusals(name):
    tensors = ("x", "residual", "sum", "y") if name == "fwd" else ("dy", "dsum", "s", "dx", "dresidual")
    for what in ("x", "y") if name == "fwd" else ("dy", "s", "saved"):
        assert _norm(name, **{what: None}) == NULL, what
    for what, value in (("M", 0), ("M", 1 << 31), ("C", 0), ("C", -1), ("C", 32769), ("C", 1 << 40)):
        assert _norm(name, **{what: value}) == DIM, (what, value)
    for what in tensors + (("weight", "bias") if name == "fwd" else ("weight", "dweight", "dbias")):
        assert _norm(name, **{what: ODD}) == ALIGN, what
    assert _norm(name, saved=C.c_void_p(0x10004)) == ALIGN
    assert _norm(name, dtype=3) == DTYPE and _norm(name, pdtype=3) == DTYPE
    assert _norm(name, dropout=_drop(2.0)) == OPTION
    if name == "fwd":
        for eps in (-1e-5, float("nan"), float("inf")):
            assert _norm(name, eps=eps) == OPTION
    else:
        assert _norm(name, dx=None, dresidual=None, dweight=None, dbias=None) == NULL
        assert _norm(name, ws=None) == WORKSPACE and _norm(name, bytes=16) == WORKSPACE and _norm(name, ws=C.c_void_p(0x10008)) == ALIGN


def test_layernorm_sizes():
    size = B.load().hdqt_layernorm_bwd_workspace_size
    assert size(0, 64, 0) == 0 and size(10, 32769, 0) == 0 and size(10, 64, 4) == 0
    assert 0 < size(10, 64, 0) <= 1 << 16
    # parts of the parameters' gradients: of as many workgroups as the chip holds, however many rows
    assert size(1 << 30, 4096, 1) <= 1024 * 2 * 4096 * 4


def _adapt(name, **changes):
    lib = B.load()
    sizes = dict(M=100, K=64, N=96, r=8, n=4, dtype=0)
    if name == "fwd":
        return lib.hdqt_adapters_fwd(*_with({**dict(x=FAKE, A=FAKE, B=FAKE, ids=FAKE, scale=FAKE, base=FAKE, out=FAKE, saved=FAKE, saved_bytes=1 << 40),
                                             **sizes, "stream": None}, **changes))
    return lib.hdqt_adapters_bwd(*_with({**dict(dy=FAKE, x=FAKE, A=FAKE, B=FAKE, ids=FAKE, scale=FAKE, saved=FAKE, saved_bytes=1 << 40, base=FAKE,
                                                dx=FAKE, dA=FAKE, dB=FAKE), **sizes, "ws": FAKE, "bytes": 1 << 40, "stream": None}, **changes))


@pytest.mark.parametrize("name", ["fwd", "bwd"])
def test_adapters_refusals(name):
    for what in ("x", "A", "B", "ids", "saved") + (("out",) if name == "fwd" else ("dy",)):
        assert _adapt(name, **{what: None}) == NULL, what
    for what, value in (("M", 0), ("M", 65535 * 64 + 1), ("K", 0), ("K", (1 << 21) + 1), ("N", -1), ("N", (1 << 21) + 1), ("r", 0), ("r", 129),
                        ("n", 0), ("n", 1025)):
        assert _adapt(name, **{what: value}) == DIM, (what, value)
    for what in ("x", "A", "B", "ids", "scale", "base", "saved") + (("out",) if name == "fwd" else ("dy", "dx", "dA", "dB")):
        assert _adapt(name, **{what: ODD}) == ALIGN, what
    assert _adapt(name, dtype=2) == DTYPE and _adapt(name, saved_bytes=16) == WORKSPACE
    if name == "bwd":
        assert _adapt(name, dx=None, dA=None, dB=None) == NULL
        assert _adapt(name, ws=None) == WORKSPACE and _adapt(name, bytes=16) == WORKSPACE and _adapt(name, ws=C.c_void_p(0x10008)) == ALIGN


def test_adapters_sizes():
    lib = B.load()
    for f in (lib.hdqt_adapters_saved_size, lib.hdqt_adapters_bwd_workspace_size):
        assert f(0, 64, 64, 8, 4, 0) == 0 and f(10, 64, 64, 129, 4, 0) == 0 and f(10, 64, 64, 8, 1025, 0) == 0 and f(10, 64, 64, 8, 4, 7) == 0
        assert 0 < f(10, 64, 64, 8, 4, 0) < 1 << 16
        # h in 32 bits of at most four parts, a plan, and sums of the gradients of at most 1024 workgroups
        assert f(1 << 20, 4096, 4096, 16, 8, 1) < (1 << 20) * 16 * 4 + (1 << 23) + 16 * 8 * 16 * 8192 * 4


def test_binding_refuses_other_forms():
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    d = B.Dropout(0.5)
    for call in (lambda: B.dropout(x, d), lambda: B.layernorm_fwd(x), lambda: B.layernorm_fwd(x, dropout=d),
                 lambda: B.layernorm_bwd(x, x, torch.zeros(4, 2)), lambda: B.adapters_fwd(x, torch.zeros(2, 8, 3), torch.zeros(2, 3, 5), ids)):
        with pytest.raises(ValueError):
            call()


def test_modules_refuse():
    with pytest.raises(ValueError):
        A.ResidualDropout(1.5)
    with pytest.raises(ValueError):
        A.ResidualNorm(8, p=-0.1)
    with pytest.raises(ValueError):
        A.HdqtLinear(8, 8)(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64))


def test_masks_move_on_in_training_alone():
    m = A.ResidualDropout(0.5, seed=10, layer_id=3)
    first, second = m.masks.next(True), m.masks.next(True)
    assert (first.seed, second.seed, first.tensor_id) == (10, 11, 3) and m.masks.next(False) is None
    m.masks.counter = torch.zeros(1, dtype=torch.int64)
    third, fourth = m.masks.next(True), m.masks.next(True)
    assert third.seed == fourth.seed == 12 and third.step is m.masks.counter
    assert A.ResidualDropout(0.0).masks.next(True) is None
    x = torch.ones(3)
    assert A.ResidualDropout(0.5).eval()(x) is x
