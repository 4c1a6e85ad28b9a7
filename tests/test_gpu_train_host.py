"""The operators around the products through the native marshalling and through ctypes: the same results and the same
refusals."""
import math

import pytest
import torch

from paper_2310_03675_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _calls():
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s, dtype=F32: torch.randn(s, generator=g, device="cuda", dtype=dtype)
    X, W, b = new(40, 24), new(24, 60)[:, :50], new(50)
    t = torch.randint(0, 50, (40,), device="cuda", generator=g)
    x, dy, w = new(3, 5, 7, 16), new(3, 5, 7, 16), torch.nn.Parameter(new(16))
    grads = [new(7, 9), new(100, dtype=BF16), new(0)]

    def norm(**k):
        y, saved = B.groupnorm_fwd(x, 4, w, new(16) * 0, **k)
        return (y, saved) + B.groupnorm_bwd(dy, x, saved, 4, w, None, need=(True, False, True))

    def clip(kind=2.0, out=False):
        v = [q.clone() for q in grads]
        o = [torch.zeros_like(q) for q in v] if out else None
        return (B.clip_grad_norm(v, 0.3, norm_type=kind, out=o),) + tuple(v) + tuple(o or ())

    def bwd(dloss, reduction, **k):
        saved = B.xent_fwd(X, W, t, b, reduction=reduction)[1]
        return B.xent_bwd(dloss, X, W, t, saved, b, reduction=reduction, **k)

    ok = [lambda: B.xent_fwd(X, W, t), lambda: B.xent_fwd(X, W, t, b, reduction="none"), lambda: B.xent_step(X, W, t, b, ignore_index=3),
          lambda: B.xent_step(X.to(BF16), W.to(BF16), t, b, reduction="sum"), lambda: B.xent_step(X, W, t, need=(False, True, False)),
          lambda: bwd(None, "mean"), lambda: bwd(torch.full((), 2.0, device="cuda"), "sum"), lambda: bwd(new(40) * 0 + 3, "none"),
          lambda: bwd(None, "none", need=(True, False, False)), norm, lambda: norm(act="relu", eps=1e-3),
          lambda: B.groupnorm_fwd(x.to(BF16), 16, act="silu"), clip, lambda: clip(math.inf, True),
          lambda: (B.grad_norm(grads), B.grad_norm(tuple(grads), math.inf))]
    refused = [lambda: B.xent_fwd(X, W, t, b, reduction="most"), lambda: B.xent_fwd(X.t(), W, t), lambda: B.xent_fwd(X, W, t, X),
               lambda: B.xent_fwd(X, W, t.cpu()), lambda: B.xent_step(X, W, t, need=(False, False, False)),
               lambda: bwd(new(40), "mean"), lambda: B.groupnorm_fwd(x, 5), lambda: B.groupnorm_fwd(x, 4, eps=-1.0),
               lambda: B.groupnorm_fwd(x, 4, act="gelu"), lambda: B.groupnorm_fwd(x.transpose(0, 1), 4),
               lambda: B.groupnorm_bwd(dy, x, x, 4), lambda: B.clip_grad_norm(grads, -1.0), lambda: B.clip_grad_norm(grads, 1.0, eps=math.nan),
               lambda: B.clip_grad_norm([X.double()], 1.0), lambda: B.clip_grad_norm([W], 1.0), lambda: B.clip_grad_norm([], 1.0),
               lambda: B.clip_grad_norm(grads, 1.0, out=grads[:2]), lambda: B.grad_norm(grads, 3.0)]
    return ok, refused


def _outcomes(calls):
    got = []
    for call in calls:
        try:
            r = call()
            got.append(tuple(None if v is None else v.clone() for v in (r if isinstance(r, tuple) else (r,))))
        except (ValueError, B.HdqtError) as e:
            got.append((type(e), str(e)))
    return got


def test_native_and_ctypes_agree(monkeypatch):
    assert not isinstance(B._host, B._LongWay)
    native = [_outcomes(c) for c in _calls()]
    monkeypatch.setattr(B, "_host", B._LongWay())
    long = [_outcomes(c) for c in _calls()]
    for a, b in zip(native[0], long[0]):
        assert len(a) == len(b)
        assert all(p is q is None or (p.dtype == q.dtype and p.shape == q.shape and torch.equal(p, q)) for p, q in zip(a, b))
    assert native[1] == long[1] and all(isinstance(r[0], type) for r in native[1])


def test_ordinary_calls_are_native():
    ok, _ = _calls()

    class Only:
        """The native functions, whose refusal to take a call is an error here."""
        def __init__(self, of):
            self.of = of

        def __getattr__(self, name):
            f = getattr(self.of, name)

            def call(*args):
                r = f(*args)
                assert r is not None, name
                return r
            return call

    host = B._host
    B._host = Only(host)
    try:
        _outcomes(ok)
    finally:
        B._host = host
