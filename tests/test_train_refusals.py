"""Calls of the operators around the products that are refused: on the host, before anything is launched (no GPU)."""
import ctypes as C

import pytest
import torch

from paper_2310_03675_amd import binding as B

FAKE = C.c_void_p(0x10000)
ODD = C.c_void_p(0x10001)
NULL, DIM, WORKSPACE, ALIGN, DTYPE, OPTION = -1, -2, -10, -11, -15, -16


def _with(ok, **changes):
    return tuple({**ok, **changes}.values())


def _xent(name, **changes):
    lib = B.load()
    ok = dict(X=FAKE, ldx=64, W=FAKE, ldw=100, bias=FAKE, target=FAKE, ignore=-100, M=32, K=64, N=100, dtype=0, bias_dtype=0,
              reduction=1)
    grads = dict(dX=FAKE, dW=FAKE, dbias=FAKE)
    end = dict(ws=FAKE, bytes=1 << 40, stream=None)
    if name == "fwd":
        return lib.hdqt_xent_fwd(*_with({**ok, "loss": FAKE, "saved": FAKE, **end}, **changes))
    if name == "bwd":
        return lib.hdqt_xent_bwd(*_with({"dloss": FAKE, **ok, "saved": FAKE, **grads, **end}, **changes))
    return lib.hdqt_xent_step(*_with({**ok, "loss": FAKE, "saved": FAKE, **grads, **end}, **changes))


@pytest.mark.parametrize("name", ["fwd", "bwd", "step"])
def test_xent_refusals(name):
    for what in ("X", "W", "target", "saved"):
        assert _xent(name, **{what: None}) == NULL, what
    for what, value in (("M", 0), ("K", 0), ("N", -1), ("M", 1 << 23), ("K", (1 << 21) + 1), ("ldx", 63), ("ldw", 99), ("ldw", 1 << 50)):
        assert _xent(name, **{what: value}) == DIM, (what, value)
    for what in ("X", "W", "bias", "target", "saved"):
        assert _xent(name, **{what: ODD}) == ALIGN, what
    assert _xent(name, dtype=2) == DTYPE and _xent(name, bias_dtype=-1) == DTYPE
    assert _xent(name, reduction=3) == OPTION
    assert _xent(name, ws=None) == WORKSPACE and _xent(name, bytes=16) == WORKSPACE
    assert _xent(name, ws=C.c_void_p(0x10010)) == ALIGN
    if name != "bwd":
        assert _xent(name, loss=None) == NULL and _xent(name, loss=ODD) == ALIGN
    if name != "fwd":
        assert _xent(name, dX=None, dW=None, dbias=None) == NULL
        assert _xent(name, dX=ODD) == ALIGN and _xent(name, dW=ODD) == ALIGN and _xent(name, dbias=ODD) == ALIGN


def test_xent_sizes():
    lib = B.load()
    assert lib.hdqt_xent_saved_size(0) == 0 and lib.hdqt_xent_saved_size(7) >= 28
    for f in (lib.hdqt_xent_fwd_workspace_size, lib.hdqt_xent_bwd_workspace_size, lib.hdqt_xent_step_workspace_size):
        assert f(0, 64, 100, 0) == 0 and f(32, 64, 100, 5) == 0 and f(1 << 23, 64, 100, 0) == 0
        assert 0 < f(32, 64, 100, 0) < 1 << 20
    # what the backward call holds does not grow with the logits
    assert lib.hdqt_xent_bwd_workspace_size(8192, 4096, 1 << 20, 1) < 1 << 30


def _norm(name, **changes):
    lib = B.load()
    sizes = dict(B=2, P=16, C=64, G=8)
    end = dict(act=0, dtype=0, pdtype=0, ws=FAKE, bytes=1 << 40, stream=None)
    if name == "fwd":
        return lib.hdqt_groupnorm_fwd(*_with({**dict(x=FAKE, weight=FAKE, bias=FAKE, y=FAKE, saved=FAKE), **sizes,
                                              "eps": 1e-5, **end}, **changes))
    return lib.hdqt_groupnorm_bwd(*_with({**dict(dy=FAKE, x=FAKE, weight=FAKE, bias=FAKE, saved=FAKE, dx=FAKE, dweight=FAKE,
                                                 dbias=FAKE), **sizes, **end}, **changes))


@pytest.mark.parametrize("name", ["fwd", "bwd"])
def test_groupnorm_refusals(name):
    for what in ("x", "saved") + (("y",) if name == "fwd" else ("dy",)):
        assert _norm(name, **{what: None}) == NULL, what
    for what, value in (("B", 0), ("P", 0), ("C", 0), ("G", 0), ("G", 7), ("G", 128), ("B", 65536), ("C", 65537), ("P", 1 << 31)):
        assert _norm(name, **{what: value}) == DIM, (what, value)
    for what in ("x", "weight", "bias", "saved") + (("y",) if name == "fwd" else ("dy", "dx", "dweight", "dbias")):
        assert _norm(name, **{what: ODD}) == ALIGN, what
    assert _norm(name, dtype=3) == DTYPE and _norm(name, pdtype=3) == DTYPE and _norm(name, act=3) == OPTION
    assert _norm(name, ws=None) == WORKSPACE and _norm(name, bytes=16) == WORKSPACE
    if name == "fwd":
        for eps in (-1e-5, float("nan"), float("inf")):
            assert _norm(name, eps=eps) == OPTION
    else:
        assert _norm(name, dx=None, dweight=None, dbias=None) == NULL
    assert B.load().hdqt_groupnorm_workspace_size(2, 16, 64, 7, 0, 1) == 0


def _rows(*rows):
    return (B.CTensor * len(rows))(*(B.CTensor(*r) for r in rows))


def test_clip_refusals():
    lib = B.load()
    a, ok = 0x10000, (0x10000, 0x20000, 100, 0, 0)
    clip = lambda rows, n=None, norm=FAKE, most=1.0, eps=1e-6, kind=0, ws=FAKE, size=1 << 30: lib.hdqt_clip_grad_norm(
        rows, len(rows) if n is None else n, most, eps, kind, norm, ws, size, None)
    assert clip(_rows(ok), norm=None) == NULL
    assert clip(_rows((0, a, 1, 0, 0))) == NULL and clip(_rows((a, 0, 1, 0, 0))) == NULL
    assert lib.hdqt_clip_grad_norm(None, 1, 1.0, 0.0, 0, FAKE, FAKE, 1 << 30, None) == NULL
    assert clip(_rows((a, a, -1, 0, 0))) == DIM and clip(_rows((a, a, 1 << 40, 0, 0))) == DIM and clip(_rows(ok), n=-1) == DIM
    assert clip(_rows((a, a, 1, 2, 0))) == DTYPE
    assert clip(_rows((a + 2, a, 1, 0, 0))) == ALIGN and clip(_rows((a + 1, a, 1, 1, 0))) == ALIGN
    assert clip(_rows(ok), norm=C.c_void_p(0x10002)) == ALIGN
    for most in (-1.0, float("nan")):
        assert clip(_rows(ok), most=most) == OPTION
    assert clip(_rows(ok), eps=-1.0) == OPTION and clip(_rows(ok), kind=2) == OPTION
    assert clip(_rows(ok), ws=None) == WORKSPACE and clip(_rows(ok), size=8) == WORKSPACE
    assert lib.hdqt_grad_norm(_rows((a + 2, 0, 1, 0, 0)), 1, 0, FAKE, FAKE, 1 << 30, None) == ALIGN
    size = lib.hdqt_clip_grad_norm_workspace_size
    assert size(_rows((a, a, -1, 0, 0)), 1) == 0 and 0 < size(_rows(ok), 1) < 1 << 16
    assert size(_rows((a, a, (1 << 40) - 1, 0, 0)), 1) < 1 << 20           # (one number for a piece, whose length grows)


def test_binding_refuses_other_forms():
    x, w, t = torch.zeros(4, 8), torch.zeros(8, 10), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: B.xent_fwd(x, w, t), lambda: B.groupnorm_fwd(x, 2), lambda: B.clip_grad_norm([x], 1.0),
                 lambda: B.clip_grad_norm([], 1.0), lambda: B.grad_norm([x])):
        with pytest.raises(ValueError):
            call()
