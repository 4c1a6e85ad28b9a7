"""A residual block's operators through the native marshalling and through ctypes: the same results and the same refusals."""
import math

import pytest
import torch

from paper_2310_03675_amd import binding as B
from test_gpu_train_host import _outcomes

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _calls():
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s, dtype=F32: torch.randn(s, generator=g, device="cuda", dtype=dtype)
    x, r, dy, w, b = new(6, 7, 40), new(6, 7, 40), new(6, 7, 40), torch.nn.Parameter(new(40)), new(40)
    d = B.Dropout(0.25, 2 ** 64 - 5, 9, torch.full((1,), 3, dtype=torch.int64, device="cuda"))
    h, A, Bm, base = new(30, 24), new(4, 24, 5), new(4, 5, 50), new(30, 50)
    ids, scale = torch.randint(-1, 4, (30,), device="cuda", generator=g), new(4)
    room, side = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def norm(wt=w, bs=b, need=(True,) * 4, t=F32, back={}, **k):
        y, s, saved = B.layernorm_fwd(x.to(t), wt, bs, **{q: v.to(t) if isinstance(v, torch.Tensor) else v for q, v in k.items()})
        return (y, s, saved) + B.layernorm_bwd(dy.to(t), s, saved, wt, dropout=k.get("dropout"), need=need, **back)

    def adapt(t=F32, need=(True,) * 3, back={}, **k):
        k = {q: v.to(t) if q == "base" else v for q, v in k.items()}
        out, saved = B.adapters_fwd(h.to(t), A.to(t), Bm.to(t), ids, **k)
        return (out,) + B.adapters_bwd(base.to(t), h.to(t), A.to(t), Bm.to(t), ids, saved, scale=k.get("scale"), need=need, **back)

    ok = [lambda: B.dropout(x, d), lambda: B.dropout(x, B.Dropout(1, -7, -1), residual=r), lambda: B.dropout(x, d, out=x.clone()),
          norm, lambda: norm(eps=1e-3, residual=r, dropout=d), lambda: norm(None, None, t=BF16, dropout=d, need=(False, True, True, False)),
          lambda: norm(residual=r, need=(True, True, False, False), back={"dsum": r}), lambda: norm(w.detach().to(BF16), b.to(BF16), t=BF16),
          lambda: B.layernorm_fwd(x, bias=b, residual=r, need=(False, False)), lambda: B.layernorm_fwd(x[0, 0]),
          adapt, lambda: adapt(scale=scale, base=base, need=(True, False, True)), lambda: adapt(BF16, base=base, back={"base": h.to(BF16)}),
          lambda: adapt(base=base, out=base.clone())]
    other = [lambda: B.layernorm_fwd(x, w, b, out=torch.empty_like(x)), lambda: norm(back={"workspace": room}), lambda: adapt(back={"workspace": room}),
             lambda: adapt(back={"out": torch.empty_like(h)})]
    refused = [lambda: B.dropout(x, None), lambda: B.dropout(x, B.Dropout(2.0)), lambda: B.dropout(x, B.Dropout(math.nan)),
               lambda: B.dropout(x.transpose(0, 1), d), lambda: B.dropout(x, d, residual=r[0]), lambda: B.dropout(x.double(), d),
               lambda: B.dropout(x[:0], d), lambda: B.dropout(x, B.Dropout(0.5, step=torch.zeros(1, dtype=torch.int64))),
               lambda: B.dropout(x, B.Dropout(0.5, step=torch.zeros(2, dtype=torch.int64, device="cuda"))),
               lambda: B.layernorm_fwd(x, w[:-1]), lambda: B.layernorm_fwd(x, w, b.to(BF16)), lambda: B.layernorm_fwd(x, eps=-1.0),
               lambda: B.layernorm_fwd(x.transpose(0, 1)), lambda: B.layernorm_fwd(x, residual=r.to(BF16)), lambda: B.layernorm_fwd(new(1, 32769)),
               lambda: B.layernorm_bwd(dy, x, x), lambda: norm(need=(False,) * 4), lambda: norm(back={"dsum": r[0]}),
               lambda: B.adapters_fwd(h, A, Bm, ids[:-1]), lambda: B.adapters_fwd(h, A[:, :-1], Bm, ids), lambda: B.adapters_fwd(h, A, Bm[:2], ids),
               lambda: B.adapters_fwd(h, A.to(BF16), Bm, ids), lambda: B.adapters_fwd(h, A, Bm, ids.int()), lambda: B.adapters_fwd(h, A, Bm, ids.cpu()),
               lambda: B.adapters_fwd(h, A, Bm, ids, scale=scale.to(BF16)), lambda: B.adapters_fwd(h, A, Bm, ids, base=base.t()),
               lambda: B.adapters_fwd(h, new(4, 24, 129), new(4, 129, 50), ids), lambda: adapt(need=(False,) * 3),
               lambda: B.adapters_bwd(base, h, A, Bm, ids, room[:16]), lambda: B.adapters_bwd(base, h, A, Bm, ids, h),
               lambda: B.adapters_bwd(h, h, A, Bm, ids, room)]
    return ok, other, refused


def test_native_and_ctypes_agree(monkeypatch):
    assert not isinstance(B._host, B._LongWay)
    native = [_outcomes(c) for c in _calls()]
    monkeypatch.setattr(B, "_host", B._LongWay())
    long = [_outcomes(c) for c in _calls()]
    for way in (0, 1):
        for a, b in zip(native[way], long[way]):
            assert len(a) == len(b)
            assert all(p is q is None or (p.dtype == q.dtype and p.shape == q.shape and torch.equal(p, q)) for p, q in zip(a, b))
    assert native[2] == long[2] and all(isinstance(r[0], type) for r in native[2])


def test_ordinary_calls_are_native():
    ok = _calls()[0]

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
