"""The operators of a residual block around an adapted layer: layer normalisation with the residual sum in front of it, dropout
from a counter-based generator, and low-rank adapters beside a shared projection, in a plain form (elementary torch operations in
32 bits) and as the library's calls.

listed()   the fixed cases; the comment at each says what it stands for
draw(rng)  one more case of the same ranges
prepare    what a program has in hand before the call
run        one pass, plain or by the library (`own`)
exact      the same outputs from the definition in 64 bits
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


def _norm(name, what, M, C, dtype, residual=False, p=0.0, affine="float32"):
    """Layer normalisation of M rows of C, of x itself or of residual + dropout(x).  what: "step" (forward and backward, with a
    gradient that reaches the sum from elsewhere where there is a residual) or "fwd".  affine: the type of weight and bias, or
    "none"."""
    return {"name": name, "op": "layernorm", "what": what, "M": M, "C": C, "dtype": dtype, "residual": residual, "p": p,
            "affine": affine}


def _drop(name, M, C, dtype, p, residual=False):
    """Dropout of a tensor, added to a residual or not, and its gradient: the same mask again."""
    return {"name": name, "op": "dropout", "what": "step", "M": M, "C": C, "dtype": dtype, "p": p, "residual": residual}


def _adapt(name, what, M, K, N, r, n, dtype, none=0.0, order="mixed"):
    """n adapters of rank r beside a projection of K features to N: M rows, each with an adapter of its own, a share `none` of
    them without.  order: "mixed" (a training batch that mixes tasks) or "runs" (requests of many rows one after the other)."""
    return {"name": name, "op": "adapters", "what": what, "M": M, "K": K, "N": N, "r": r, "n": n, "dtype": dtype, "none": none,
            "order": order}


def listed():
    return [
        # a single sample of the sensor network (561 features): all latency
        _norm("norm_1x561", "fwd", 1, 561, "float32"),
        # the features in front of ResNet-18's classifier at its batch of 128, a residual block around them
        _norm("norm_128x512", "step", 128, 512, "float32", residual=True, p=0.1),
        # every pixel of ResNet-18's first stage at that batch: many short rows
        _norm("norm_131072x64", "step", 131072, 64, "float32"),
        # odd rows and columns
        _norm("norm_20011x1031", "step", 20011, 1031, "bfloat16", residual=True),
        # a block's end in training, 8192 tokens of 4096
        _norm("norm_8192x4096", "step", 8192, 4096, "bfloat16", residual=True, p=0.1, affine="bfloat16"),
        # those 128 rows of features dropped out alone: all latency
        _drop("dropout_128x512", 128, 512, "float32", 0.5),
        # the operand of the benchmark's layer
        _drop("dropout_65536x1152", 65536, 1152, "float32", 0.1, residual=True),
        # one sample of the sensor network through one of ten tasks' adapters
        _adapt("adapt_1x561x512_r8", "fwd", 1, 561, 512, 8, 10, "float32"),
        # 32 requests that each answer their next token, 64 adapters loaded
        _adapt("adapt_32x4096x4096_r16", "fwd", 32, 4096, 4096, 16, 64, "bfloat16"),
        # a batch of 128 that mixes ten tasks, in training
        _adapt("adapt_128x512x512_r8", "step", 128, 512, 512, 8, 10, "float32", none=0.1),
        # odd sizes, a rank that is no power of two, some rows without an adapter
        _adapt("adapt_4999x1153x2311_r24", "step", 4999, 1153, 2311, 24, 17, "float32", none=0.15),
        # a large training batch, and the largest: 8192 tokens in 32 requests
        _adapt("adapt_8192x4096x16384_r64", "step", 8192, 4096, 16384, 64, 32, "bfloat16", order="runs"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["layernorm", "layernorm", "dropout", "adapters", "adapters"])
    dtype = rng.choice(["float32", "bfloat16"])
    if op == "layernorm":
        C = 2 ** rng.randint(3, 14) if rng.random() < 0.4 else _log(rng, 8, 30000)
        M = min(_log(rng, 1, 200000), max(1, 33_000_000 // C))
        # (a bfloat16 sum within a rounding in 32 bits of the middle between two values has two right ones, which a gradient of
        # the parameters in 32 bits would show: behind dropout's product they are of the tensors' type)
        p = rng.choice([0.0, 0.1, 0.37])
        return {"op": op, "what": rng.choice(["step", "step", "fwd"]), "M": M, "C": C, "dtype": dtype, "residual": rng.random() < 0.6,
                "p": p, "affine": rng.choice(["none", dtype, dtype, dtype if p else "float32"])}
    if op == "dropout":
        C = _log(rng, 1, 8192)
        return {"op": op, "what": "step", "M": min(_log(rng, 1, 1_000_000), max(1, 75_000_000 // C)), "C": C, "dtype": dtype,
                "p": rng.choice([0.1, 0.5, round(rng.uniform(0.01, 0.9), 3)]), "residual": rng.random() < 0.5}
    M, K, N = _log(rng, 1, 8192), _log(rng, 64, 8192), _log(rng, 64, 8192)
    if rng.random() < 0.5:
        K, N = 2 ** rng.randint(6, 13), 2 ** rng.randint(6, 13)
    return {"op": op, "what": rng.choice(["step", "fwd"]), "M": M, "K": K, "N": N,
            "r": rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 64)]), "n": _log(rng, 1, 64), "dtype": dtype,
            "none": rng.choice([0.0, 0.0, 0.2]), "order": rng.choice(["mixed", "runs"])}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 29)
    dt = DTYPES[case["dtype"]]

    def normal(shape, std=1.0, mean=0.0, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)

    state = {"case": case, "seed": int(seed) * 2654435761 % 2 ** 64, "id": 7}
    if case["op"] == "adapters":
        M, K, N, r, n = (case[k] for k in ("M", "K", "N", "r", "n"))
        ids = torch.randint(0, n, (M,), device="cuda", generator=g)
        if case["order"] == "runs":
            ids = torch.sort(ids)[0]
            ids = torch.randperm(n, device="cuda", generator=g)[ids]
        drop = torch.rand(M, device="cuda", generator=g) < case["none"]
        state.update(x=normal((M, K)), base=normal((M, N)), A=normal((n, K, r), 1 / math.sqrt(K)), B=normal((n, r, N), 1 / math.sqrt(r)),
                     ids=torch.where(drop, torch.full_like(ids, -1), ids),
                     scale=torch.rand(n, device="cuda", generator=g) + 0.5)
        if case["what"] == "step":
            state["dy"] = normal((M, N))
        return state
    M, C = case["M"], case["C"]
    state["x"] = normal((M, C), 1.5, 0.3)
    if case["residual"]:
        state["residual"] = normal((M, C), 1.0, 0.1)
    if case["op"] == "layernorm" and case["affine"] != "none":
        state.update(weight=normal((C,), 0.2, 1.0, DTYPES[case["affine"]]), bias=normal((C,), 0.2, 0.0, DTYPES[case["affine"]]))
    if case["what"] == "step":
        state["dy"] = normal((M, C))
        if case["op"] == "layernorm" and case["residual"]:
            state["dsum"] = normal((M, C))
    return state


def _philox(block, word3, seed, tensor_id):
    """Four words of 32 bits for each block's number, in 64-bit integers: counter (block, tensor id, word3), ten rounds."""
    low = 0xFFFFFFFF
    c0, c1 = block & low, block >> 32
    c2, c3 = torch.full_like(block, tensor_id), torch.full_like(block, word3)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), 1)


def _threshold(p):
    return int(round(p * 2 ** 32))


def _kept(s, n):
    """Which of n elements are kept: element e has the 16-bit field e mod 8 of block e / 8, and 16 bits more below it."""
    block = torch.arange((n + 7) // 8, device="cuda")
    high, low = (_philox(block, w, s["seed"], s["id"]) for w in (1, 2))
    fields = lambda words: torch.stack((words & 0xFFFF, words >> 16), 2).reshape(-1)[:n]
    return (fields(high) << 16) + fields(low) >= _threshold(s["case"]["p"])


def _dropped(s, v, kept):
    if kept is None:
        return v
    t = _threshold(s["case"]["p"])
    return torch.where(kept, v * (2 ** 32 / (2 ** 32 - t)), torch.zeros_like(v))


def _plain_drop(s):
    case, x = s["case"], s["x"]
    kept = _kept(s, x.numel()).reshape(x.shape)
    y = _dropped(s, x.float(), kept)
    if case["residual"]:
        y = s["residual"].float() + y
    return {"y": y.to(x.dtype), "dx": _dropped(s, s["dy"].float(), kept).to(x.dtype)}


def _plain_norm(s):
    case, x, dt = s["case"], s["x"].float(), s["x"].dtype
    kept = _kept(s, x.numel()).reshape(x.shape) if case["p"] else None
    out = {}
    v = _dropped(s, x, kept)
    if case["residual"]:
        v = s["residual"].float() + v
    if case["residual"] or case["p"]:
        out["sum"] = v.to(dt)               # the sum is a tensor of the network, and what is normalised
        v = out["sum"].float()
    mean = v.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    xh = (v - mean) * rstd
    affine = case["affine"] != "none"
    out["y"] = (xh * s["weight"].float() + s["bias"].float() if affine else xh).to(dt)
    if case["what"] == "step":
        d = s["dy"].float()
        if affine:
            out["dweight"], out["dbias"] = (v.to(s["weight"].dtype) for v in ((d * xh).sum(0), d.sum(0)))
            d = d * s["weight"].float()
        ds = rstd * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
        if case["residual"]:
            ds = ds + s["dsum"].float()
            out["dresidual"] = ds.to(dt)
        out["dx"] = _dropped(s, ds, kept).to(dt)
    return out


def _plain_adapters(s):
    case, dt = s["case"], s["x"].dtype
    M, K, N, r, n = (case[k] for k in ("M", "K", "N", "r", "n"))
    # every row through all adapters at once, and what is not of its own set to zero
    x, A, B = s["x"].float(), s["A"].float().permute(1, 0, 2).reshape(K, n * r), s["B"].float().reshape(n * r, N)
    mine = (s["ids"][:, None] == torch.arange(n, device="cuda")).repeat_interleave(r, 1)
    scale = s["scale"].repeat_interleave(r)
    zero = torch.zeros((), device="cuda")
    H = torch.where(mine, (x @ A) * scale, zero)
    out = {"out": (s["base"].float() + H @ B).to(dt)}
    if case["what"] == "step":
        dy = s["dy"].float()
        dH = torch.where(mine, (dy @ B.t()) * scale, zero)
        out["dx"] = (dH @ A.t()).to(dt)
        out["dA"] = (x.t() @ dH).reshape(K, n, r).permute(1, 0, 2).to(dt)
        out["dB"] = (H.t() @ dy).reshape(n, r, N).to(dt)
    return out


def _own_run(s):
    from paper_2310_03675_amd import binding as B

    case = s["case"]
    if case["op"] == "adapters":
        y, saved = B.adapters_fwd(s["x"], s["A"], s["B"], s["ids"], scale=s["scale"], base=s["base"])
        out = {"out": y}
        if case["what"] == "step":
            out["dx"], out["dA"], out["dB"] = B.adapters_bwd(s["dy"], s["x"], s["A"], s["B"], s["ids"], saved, scale=s["scale"])
        return out
    drop = B.Dropout(p=case["p"], seed=s["seed"], tensor_id=s["id"]) if case["p"] else None
    if case["op"] == "dropout":
        return {"y": B.dropout(s["x"], drop, residual=s.get("residual")), "dx": B.dropout(s["dy"], drop)}
    w, b, summed = s.get("weight"), s.get("bias"), case["residual"] or drop is not None
    y, total, saved = B.layernorm_fwd(s["x"], w, b, eps=1e-5, residual=s.get("residual"), dropout=drop)
    out = {"y": y, **({"sum": total} if summed else {})}
    if case["what"] == "step":
        need = (True, case["residual"], w is not None, b is not None)
        grads = B.layernorm_bwd(s["dy"], total, saved, w, dsum=s.get("dsum"), dropout=drop, need=need)
        out.update((k, v) for k, v, wanted in zip(("dx", "dresidual", "dweight", "dbias"), grads, need) if wanted)
    return out


def run(state):
    if own:
        return _own_run(state)
    return {"layernorm": _plain_norm, "dropout": _plain_drop, "adapters": _plain_adapters}[state["case"]["op"]](state)


def work(case):
    size, step = DTYPES[case["dtype"]].itemsize, case["what"] == "step"
    if case["op"] == "adapters":
        M, K, N, r = (case[k] for k in ("M", "K", "N", "r"))
        used = min(case["n"], M) * r * (K + N) * size
        # x, base, out; a step has dy and dx besides, and the adapters' gradients
        return {"bytes": M * (K + 2 * N + (K + N if step else 0)) * size + used * (2 if step else 1) + 8 * M,
                "flops": 2 * M * r * (K + N) * (3 if step else 1)}
    n, extra = case["M"] * case["C"], 1 if case["residual"] else 0
    if case["op"] == "dropout":
        return {"bytes": n * size * (4 + extra), "flops": 2 * n * 30}
    summed = extra or case["p"] > 0
    params = 0 if case["affine"] == "none" else DTYPES[case["affine"]].itemsize * case["C"] * (4 if step else 2)
    # x, residual, the sum, y; backward dy, the sum again (it is a tensor of its own right), its gradient from elsewhere, dx, dresidual
    tensors = 2 + extra + (1 if summed else 0) + ((2 + 2 * extra) if step else 0)
    return {"bytes": n * size * tensors + params, "flops": n * (20 if step else 8)}


def _exact_kept(case, state):
    """Which elements are kept, by unsigned integers on the host; the lower 16 bits only where the upper ones leave it open."""
    n, t = case["M"] * case["C"], _threshold(case["p"])
    if t == 0:
        return torch.ones((case["M"], case["C"]), dtype=torch.bool, device="cuda")
    u64, low = np.uint64, np.uint64(0xFFFFFFFF)

    def fields(block, word3):
        c = [block & low, block >> u64(32), np.full_like(block, state["id"]), np.full_like(block, word3)]
        k = [state["seed"] & 0xFFFFFFFF, state["seed"] >> 32]
        for _ in range(10):
            a, b = c[0] * u64(0xD2511F53), c[2] * u64(0xCD9E8D57)
            c = [(b >> u64(32)) ^ c[1] ^ u64(k[0]), b & low, (a >> u64(32)) ^ c[3] ^ u64(k[1]), a & low]
            k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
        return np.stack([w for v in c for w in (v & u64(0xFFFF), v >> u64(16))], 1)

    high = np.concatenate([fields(np.arange(i, min(i + 2 ** 20, (n + 7) // 8), dtype=u64), 1).astype(np.int32)
                           for i in range(0, (n + 7) // 8, 2 ** 20)])
    keep = high > t >> 16
    for i, j in zip(*np.nonzero(high == t >> 16)):
        keep[i, j] = int(fields(np.array([i], dtype=u64), 2)[0, j]) >= t % 2 ** 16
    return torch.from_numpy(keep.reshape(-1)[:n]).cuda().reshape(case["M"], case["C"])


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["op"] == "adapters":
        out = {"out": s["base"].double()}
        if case["what"] == "step":
            out.update(dx=torch.zeros_like(x), dA=torch.zeros_like(s["A"], dtype=torch.float64), dB=torch.zeros_like(s["B"], dtype=torch.float64))
        for a in range(case["n"]):
            rows = torch.nonzero(s["ids"] == a)[:, 0]
            xa, A, B, f = x[rows], s["A"][a].double(), s["B"][a].double(), s["scale"][a].double()
            out["out"][rows] += f * torch.mm(torch.mm(xa, A), B)
            if case["what"] == "step":
                dy = s["dy"][rows].double()
                back = torch.mm(dy, B.t().contiguous())
                out["dx"][rows] = f * torch.mm(back, A.t().contiguous())
                out["dA"][a] = f * torch.mm(xa.t().contiguous(), back)
                out["dB"][a] = f * torch.mm(torch.mm(xa, A).t().contiguous(), dy)
        return out
    rate = 2.0 ** 32 / (2 ** 32 - _threshold(case["p"]))
    mask = _exact_kept(case, s) * rate
    total = torch.nan_to_num(x) * mask + (s["residual"].double() if case["residual"] else 0)
    if case["op"] == "dropout":
        return {"y": total, "dx": s["dy"].double() * mask}
    out, summed, affine = {}, case["residual"] or case["p"], case["affine"] != "none"
    if summed:
        out["sum"] = total
    v = total.to(s["x"].dtype).double().requires_grad_(case["what"] == "step")
    w, b = (s[k].double().requires_grad_() if affine else None for k in ("weight", "bias"))
    y = torch.nn.functional.layer_norm(v, (case["C"],), w, b, 1e-5)
    out["y"] = y.detach()
    if case["what"] == "step":
        grads = torch.autograd.grad(y, [v] + ([w, b] if affine else []), s["dy"].double())
        ds = grads[0] + (s["dsum"].double() if case["residual"] else 0)
        out["dx"] = ds * mask
        if case["residual"]:
            out["dresidual"] = ds
        if affine:
            out["dweight"], out["dbias"] = grads[1:]
    return out
