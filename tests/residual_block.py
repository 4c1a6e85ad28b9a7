"""What the operators of a residual block are, in 64 bits on the host, for their tests."""
import numpy as np
import torch


def fields(blocks, word3, seed, tensor_id):
    """The eight 16-bit fields of each block of Philox4x32-10: counter (block, tensor id, word3), key seed."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    b = np.asarray(blocks, dtype=u)
    c = [b & low, b >> u(32), np.full_like(b, tensor_id), np.full_like(b, word3)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(p1 >> u(32)) ^ c[1] ^ u(k0), p1 & low, (p0 >> u(32)) ^ c[3] ^ u(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack([h for w in c for h in (w & u(0xFFFF), w >> u(16))], 1).astype(np.int64)


def kept(n, p, seed, tensor_id, first=0):
    """Which of the elements first to first + n - 1 are kept."""
    blocks = np.arange(first // 8, (first + n + 7) // 8)
    draws = (fields(blocks, 1, seed % 2 ** 64, tensor_id) << 16) + fields(blocks, 2, seed % 2 ** 64, tensor_id)
    return torch.from_numpy(draws.reshape(-1)[first % 8:first % 8 + n] >= bound(p))


def bound(p):
    return round(p * 2 ** 32)


def rate(p):
    return 0.0 if bound(p) == 2 ** 32 else 2 ** 32 / (2 ** 32 - bound(p))


def dropped(x, d):
    """dropout(x) of a binding.Dropout."""
    seed = d.seed + (0 if d.step is None else int(d.step))
    mask = kept(x.numel(), d.p, seed, d.tensor_id).reshape(x.shape)
    return torch.where(mask, x.double().cpu() * rate(d.p), torch.zeros((), dtype=torch.float64))


def layer_norm(x, dy, w=None, b=None, residual=None, dsum=None, d=None, eps=1e-5, held=None):
    """Everything that the forward and the backward call give, and the sizes of what dx and dweight are sums of.  held: the sum as it
    was held (near the middle between two values of a type a sum in 32 bits may be rounded to the other one)."""
    dt = x.dtype
    v = x.double().cpu() if d is None else dropped(x, d)
    if residual is not None:
        v = residual.double().cpu() + v
    out = {"sum": v}
    C = x.shape[-1]
    v = (v.to(dt) if held is None else held.cpu()).double().reshape(-1, C)
    w = torch.ones(C, dtype=torch.float64) if w is None else w.double().cpu()
    b = torch.zeros(C, dtype=torch.float64) if b is None else b.double().cpu()
    mean = v.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((v - mean).square().mean(1, keepdim=True) + eps)
    xh = (v - mean) * rstd
    g = dy.double().cpu().reshape(-1, C)
    wd = g * w
    ds = rstd * (wd - wd.mean(1, keepdim=True) - xh * (wd * xh).mean(1, keepdim=True))
    more = 0 if dsum is None else dsum.double().cpu().reshape(-1, C)
    ds = ds + more
    out.update(y=(xh * w + b).reshape(x.shape), dresidual=ds.reshape(x.shape), dweight=(g * xh).sum(0), dbias=g.sum(0), mean=mean[:, 0],
               rstd=rstd[:, 0], ds_terms=float((rstd * wd + more).norm() + (rstd * wd).norm()),
               dw_terms=float((g * xh).square().sum().sqrt()), db_terms=float(g.square().sum().sqrt()))
    out["dx"] = out["dresidual"]
    if d is not None:
        mask = kept(x.numel(), d.p, d.seed + (0 if d.step is None else int(d.step)), d.tensor_id).reshape(x.shape)
        out["dx"] = torch.where(mask, out["dresidual"] * rate(d.p), torch.zeros((), dtype=torch.float64))
    return out


def adapters(x, A, Bm, ids, scale=None, base=None, dy=None, dbase=None):
    """out, and with dy dx, dA and dB.  Rows of numbers that are none are NaN."""
    x, A, Bm, ids = (t.cpu() for t in (x, A, Bm, ids))
    n, K, r = A.shape
    N = Bm.shape[2]
    f = torch.ones(n, dtype=torch.float64) if scale is None else scale.double().cpu()
    out = torch.zeros(x.shape[0], N, dtype=torch.float64) if base is None else base.double().cpu().clone()
    dx = torch.zeros(x.shape, dtype=torch.float64) if dbase is None else dbase.double().cpu().clone()
    dA, dB = torch.zeros(A.shape, dtype=torch.float64), torch.zeros(Bm.shape, dtype=torch.float64)
    for a in set(ids.tolist()):
        rows = (ids == a).nonzero()[:, 0]
        if a >= n:
            out[rows] = dx[rows] = float("nan")
        if a < 0 or a >= n:
            continue
        h = x[rows].double() @ A[a].double()
        out[rows] += f[a] * h @ Bm[a].double()
        if dy is not None:
            g = f[a] * dy.cpu()[rows].double() @ Bm[a].double().t()
            dx[rows] += g @ A[a].double().t()
            dA[a], dB[a] = x[rows].double().t() @ g, f[a] * h.t() @ dy.cpu()[rows].double()
    return {"out": out, "dx": dx, "dA": dA, "dB": dB}
