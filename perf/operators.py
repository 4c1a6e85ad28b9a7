"""The operators around the integer products of a training step: the classifier's loss, the
normalisation between layers and the clipping of the gradients, in a plain form (elementary torch
operations in 32 bits) and as the library's calls.

listed()   the fixed cases; the comment at each says what it stands for
draw(rng)  one more case of the same ranges
prepare    what a program has in hand before the call
run        one pass, plain or by the library (`own`)
exact      the same outputs from the definition in 64 bits
"""
import math

import torch

own = False

IGNORED = -100
DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}


def _xent(name, what, M, K, N, dtype, bias=False, ignored=0.0, spare=0, reduction="mean"):
    """The loss of a linear classifier of N classes over K features, M rows.  what: "step" (loss and
    all gradients) or "fwd" (the loss alone).  spare: classes that the weight has behind the N used
    ones (a head that grows with the tasks).  ignored: share of rows without a target."""
    return {"name": name, "op": "xent", "what": what, "M": M, "K": K, "N": N, "dtype": dtype, "bias": bias,
            "ignored": ignored, "spare": spare, "reduction": reduction}


def _norm(name, what, B, P, C, G, dtype, act):
    """Group normalisation of B images of P pixels and C channels (innermost) in G groups, with an
    activation behind it.  what: "step" (forward and backward) or "fwd"."""
    return {"name": name, "op": "groupnorm", "what": what, "B": B, "P": P, "C": C, "G": G, "dtype": dtype, "act": act}


def _clip(name, count, total, dtype, clipped=True, kind="2", sizes="mixed"):
    """Global norm of `count` gradients of about `total` elements and their clipping.  dtype may be
    "mixed" (both types in turn); clipped: whether the norm is above the limit; sizes: "resnet18"
    for that network's parameters, else drawn from the count and the total."""
    return {"name": name, "op": "clip", "count": count, "total": total, "dtype": dtype, "clipped": clipped,
            "kind": kind, "sizes": sizes}


def listed():
    return [
        # a single sample of the sensor network's classifier (561 features, 11 classes): all latency
        _xent("xent_1x561x11", "step", 1, 561, 11, "float32", bias=True),
        # the classifier of the ResNet-18 configuration at its batch of 128
        _xent("xent_128x512x100", "step", 128, 512, 100, "float32", bias=True),
        # loss of a whole test set of 10000 images, row by row, for a thousand classes
        _xent("xent_eval_10000x512x1000", "fwd", 10000, 512, 1000, "float32", bias=True, reduction="none"),
        # a head that grows: 10007 of 12000 classes in use, odd rows, every fifth without a target
        _xent("xent_grown_777x320x10007", "step", 777, 320, 10007, "float32", bias=True, ignored=0.2, spare=1993),
        # a vocabulary of odd size in bfloat16, padded sequences
        _xent("xent_4096x2048x50257", "step", 4096, 2048, 50257, "bfloat16", ignored=0.1),
        # the largest: a vocabulary of 128000, whose logits would fill 2 GB in bfloat16
        _xent("xent_8192x4096x128000", "step", 8192, 4096, 128000, "bfloat16"),
        # one small image in evaluation, odd sizes: all latency
        _norm("norm_1x49x96", "fwd", 1, 49, 96, 3, "float32", "relu"),
        # the last stage of ResNet-18 at batch 128: 4 x 4 pixels, 512 channels
        _norm("norm_128x16x512", "step", 128, 16, 512, 32, "float32", "silu"),
        # its first stage: 32 x 32 pixels, 64 channels, groups of two
        _norm("norm_128x1024x64", "step", 128, 1024, 64, 32, "float32", "silu"),
        # few large images in bfloat16, an image many times what a compute unit holds
        _norm("norm_8x65536x320", "step", 8, 65536, 320, 32, "bfloat16", "silu"),
        # the gradients of ResNet-18: 62 tensors, 64 to 2.4 million elements
        _clip("clip_resnet18", 62, 11220132, "float32", sizes="resnet18"),
        # 60 gradients of both types, 400 million elements, lengths odd and even
        _clip("clip_60x400M", 60, 400_000_000, "mixed"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["xent", "xent", "groupnorm", "groupnorm", "clip"])
    if op == "xent":
        dtype = rng.choice(["float32", "bfloat16"])
        M, K, N = _log(rng, 1, 8192), _log(rng, 32, 4096), _log(rng, 2, 128000)
        if rng.random() < 0.5:
            K = 2 ** rng.randint(5, 12)
        if dtype == "float32":                       # (the plain products run at a fraction of the bfloat16 kernels' rate)
            N = max(2, min(N, 2 ** 37 // (M * K)))
        return {"op": op, "what": rng.choice(["step", "step", "fwd"]), "M": M, "K": K, "N": N, "dtype": dtype,
                "bias": rng.random() < 0.5, "ignored": rng.choice([0.0, 0.15]),
                "spare": rng.choice([0, 0, rng.randint(1, 500)]), "reduction": rng.choice(["mean", "mean", "sum", "none"])}
    if op == "groupnorm":
        C = rng.choice([1, 2, 3, 4, 5, 8]) * rng.choice([8, 16, 24, 32, 64, 128])
        if rng.random() < 0.15:
            C = rng.randint(5, 300)
        G = rng.choice([d for d in range(1, min(C, 64) + 1) if C % d == 0])
        B, P = _log(rng, 1, 256), _log(rng, 1, 65536)
        dtype, what = rng.choice(["float32", "bfloat16"]), rng.choice(["step", "step", "fwd"])
        P = max(1, min(P, (75_000_000 if dtype == "float32" else 150_000_000) // (B * C)))
        # (behind a rectifier's jump the derivative of an element within rounding of zero has two right values)
        return {"op": op, "what": what, "B": B, "P": P, "C": C, "G": G, "dtype": dtype,
                "act": rng.choice(["none", "silu", "relu"] if what == "fwd" else ["none", "silu"])}
    return {"op": op, "count": rng.randint(1, 60), "total": _log(rng, 1000, 300_000_000),
            "dtype": rng.choice(["float32", "bfloat16", "mixed"]), "clipped": rng.random() < 0.7,
            "kind": rng.choice(["2", "2", "2", "inf"]), "sizes": "mixed"}


def _resnet18_sizes():
    def block(stage, first):
        c = 64 << stage
        cin = c // 2 if first and stage else c
        return [9 * cin * c, 9 * c * c, c, c, c, c] + ([cin * c, c, c] if first and stage else [])

    blocks = [block(stage, first) for stage in range(4) for first in (True, False)]
    return [27 * 64, 64, 64] + sum(blocks, []) + [512 * 100, 100]


def _sizes(case):
    """Lengths of a clip case's tensors, from the case alone: spread over three decades, their sum
    about the total."""
    if case["sizes"] == "resnet18":
        return _resnet18_sizes()
    w = [math.exp(6.9 * ((i * 0.6180339887) % 1.0)) for i in range(case["count"])]
    return [max(1, int(case["total"] * v / sum(w)) | (i & 1)) for i, v in enumerate(w)]


def _kinds(case):
    kinds = ["float32", "bfloat16"] if case["dtype"] == "mixed" else [case["dtype"]]
    return (kinds * case["count"])[:case["count"]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)

    def normal(shape, std=1.0, mean=0.0, dtype=torch.float32):
        # (drawn in the type itself: a large weight is not held in 32 bits on the way)
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(mean, std, generator=g)

    if case["op"] == "xent":
        M, K, N, dt = case["M"], case["K"], case["N"], DTYPES[case["dtype"]]
        X = normal((M, K), dtype=dt)
        W = normal((K, N + case["spare"]), 1.5 / math.sqrt(K), dtype=dt)[:, :N]
        bias = normal((N,), 0.5, dtype=dt) if case["bias"] else None
        t = torch.randint(0, N, (M,), device="cuda", generator=g)
        if case["ignored"]:
            drop = torch.rand(M, device="cuda", generator=g) < case["ignored"]
            drop[0] = False                          # (one row counts)
            t = torch.where(drop, torch.full_like(t, IGNORED), t)
        return {"case": case, "X": X, "W": W, "bias": bias, "t": t}
    if case["op"] == "groupnorm":
        B, P, C, dt = case["B"], case["P"], case["C"], DTYPES[case["dtype"]]
        x = normal((B, P, C), 1.5, 0.3, dtype=dt)
        x += normal((1, 1, C), dtype=dt)
        state = {"case": case, "x": x, "weight": 1 + normal((C,), 0.2), "bias": normal((C,), 0.2)}
        if case["what"] == "step":
            state["dy"] = normal((B, P, C), dtype=dt)
        return state
    grads = [normal((n,), 10.0 ** -(2 + i % 3), dtype=DTYPES[kind])
             for i, (n, kind) in enumerate(zip(_sizes(case), _kinds(case)))]
    return {"case": case, "grads": grads, "out": [torch.empty_like(v) for v in grads],
            "max_norm": 0.01 if case["clipped"] else 1e6}


def _activation(pre, act):
    """act(pre) and its derivative."""
    if act == "relu":
        return pre.clamp_min(0), (pre > 0).float()
    if act == "silu":
        s = 1 / (1 + torch.exp(-pre))
        return pre * s, s * (1 + pre * (1 - s))
    return pre, torch.ones_like(pre)


def _plain_xent(s):
    case, t = s["case"], s["t"]
    X, W, dt = s["X"].float(), s["W"].float(), s["X"].dtype
    z = X @ W
    if s["bias"] is not None:
        z = z + s["bias"].float()
    m = z.amax(1, keepdim=True)
    at = t.clamp_min(0)[:, None]
    zt = z.gather(1, at)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    keep = (t != IGNORED).float()[:, None]
    rows = keep * (m + torch.log(total) - zt)
    share = 1 / keep.sum().clamp_min(1) if case["reduction"] == "mean" else torch.ones((), device=X.device)
    out = {"loss": rows[:, 0] if case["reduction"] == "none" else rows.sum() * share}
    if case["what"] == "step":
        dz = e / total
        dz.scatter_add_(1, at, torch.full_like(zt, -1.0))
        dz = dz * (keep * share)
        out["dX"], out["dW"] = (dz @ W.t()).to(dt), (X.t() @ dz).to(dt)
        if s["bias"] is not None:
            out["dbias"] = dz.sum(0).to(dt)
    return out


def _plain_norm(s):
    case, x = s["case"], s["x"].float()
    B, P, C, G = case["B"], case["P"], case["C"], case["G"]
    x = x.reshape(B, P, G, C // G)
    w, b = s["weight"].reshape(G, C // G), s["bias"].reshape(G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean((1, 3), keepdim=True) + 1e-5)
    xh = (x - mean) * rstd
    y, slope = _activation(xh * w + b, case["act"])
    dt = s["x"].dtype
    out = {"y": y.reshape(B, P, C).to(dt)}
    if case["what"] == "step":
        d = s["dy"].float().reshape(x.shape) * slope
        out["dweight"], out["dbias"] = (d * xh).sum((0, 1)).reshape(C), d.sum((0, 1)).reshape(C)
        d = d * w
        dx = rstd * (d - d.mean((1, 3), keepdim=True) - xh * (d * xh).mean((1, 3), keepdim=True))
        out["dx"] = dx.reshape(B, P, C).to(dt)
    return out


def _plain_clip(s):
    case, grads = s["case"], s["grads"]
    flat = torch.cat([g.float() for g in grads])
    norm = flat.abs().amax() if case["kind"] == "inf" else torch.sqrt((flat * flat).sum())
    flat = flat * (s["max_norm"] / (norm + 1e-6)).clamp_max(1)
    return {"norm": norm, "grads": [v.to(g.dtype) for g, v in zip(grads, flat.split([g.numel() for g in grads]))]}


def _own_run(s):
    from paper_2310_03675_amd import binding as B

    case = s["case"]
    if case["op"] == "xent":
        kw = {"bias": s["bias"], "ignore_index": IGNORED, "reduction": case["reduction"]}
        if case["what"] == "fwd":
            return {"loss": B.xent_fwd(s["X"], s["W"], s["t"], **kw)[0]}
        loss, dX, dW, db = B.xent_step(s["X"], s["W"], s["t"], **kw)
        return {"loss": loss, "dX": dX, "dW": dW, **({} if db is None else {"dbias": db})}
    if case["op"] == "groupnorm":
        y, saved = B.groupnorm_fwd(s["x"], case["G"], s["weight"], s["bias"], eps=1e-5, act=case["act"])
        out = {"y": y}
        if case["what"] == "step":
            out["dx"], out["dweight"], out["dbias"] = B.groupnorm_bwd(s["dy"], s["x"], saved, case["G"], s["weight"],
                                                                      s["bias"], act=case["act"])
        return {k: out[k] for k in ("y", "dweight", "dbias", "dx") if k in out}
    norm = B.clip_grad_norm(s["grads"], s["max_norm"], norm_type=float(case["kind"]), eps=1e-6, out=s["out"])
    return {"norm": norm, "grads": s["out"]}


def run(state):
    if own:
        return _own_run(state)
    return {"xent": _plain_xent, "groupnorm": _plain_norm, "clip": _plain_clip}[state["case"]["op"]](state)


def work(case):
    step = case.get("what") == "step"
    if case["op"] == "xent":
        M, K, N = case["M"], case["K"], case["N"]
        size = 4 if case["dtype"] == "float32" else 2
        once = (M * K + K * N + (N if case["bias"] else 0)) * size
        loss = 4 * (M if case["reduction"] == "none" else 1)
        # (the gradients need the logits' products once: 2 MKN, and 4 MKN of their own)
        return {"bytes": once * (2 if step else 1) + 8 * M + loss, "flops": 2 * M * K * N * (3 if step else 1)}
    if case["op"] == "groupnorm":
        n, C = case["B"] * case["P"] * case["C"], case["C"]
        size = 4 if case["dtype"] == "float32" else 2
        # x in, y out; a step has dy in and dx out besides
        return {"bytes": n * size * (4 if step else 2) + 4 * C * (4 if step else 2), "flops": n * (25 if step else 10)}
    n = sum(k * DTYPES[kind].itemsize for k, kind in zip(_sizes(case), _kinds(case)))
    return {"bytes": 2 * n + 4, "flops": 3 * sum(_sizes(case))}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "xent":
        step = case["what"] == "step"
        leaf = lambda v: v.double().requires_grad_(step)
        X, W = leaf(s["X"]), leaf(s["W"])
        logits = torch.matmul(X, W)
        bias = None
        if s["bias"] is not None:
            bias = leaf(s["bias"])
            logits = logits + bias
        loss = torch.nn.functional.cross_entropy(logits, s["t"], ignore_index=IGNORED, reduction=case["reduction"])
        out = {"loss": loss.detach()}
        if step:
            grads = torch.autograd.grad(loss.sum(), [X, W] + ([] if bias is None else [bias]))
            out.update(zip(("dX", "dW", "dbias"), grads))
        return out
    if case["op"] == "groupnorm":
        step = case["what"] == "step"
        x, w, b = (s[k].double().requires_grad_(step) for k in ("x", "weight", "bias"))
        y = torch.nn.functional.group_norm(x.movedim(2, 1), case["G"], w, b, 1e-5).movedim(1, 2)
        y = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu}[case["act"]](y)
        out = {"y": y.detach()}
        if step:
            grads = torch.autograd.grad(y, [w, b, x], s["dy"].double())
            out.update(zip(("dweight", "dbias", "dx"), grads))
        return out
    p = math.inf if case["kind"] == "inf" else 2
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double(), p) for g in s["grads"]]), p)
    scale = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
    return {"norm": norm, "grads": [g.double() * scale for g in s["grads"]]}
