"""torch.autograd glue over the C ABI: a linear map Z = X W whose forward product and
both gradients are the library's quantized matmuls (Methodology: forward and
backward pass of a layer).  Nothing is computed here; the functions marshal
tensors into hdqt_layer_fwd / hdqt_layer_bwd and hand the results to autograd.

The activation is not kept in fp32 for the backward pass: hdqt_layer_fwd leaves
X's codes along the batch dimension (what the weight gradient contracts over)
in a byte buffer one eighth the size of X at 4 bits.
"""
import copy
import itertools
from dataclasses import dataclass, field
from typing import Optional

import torch

from . import binding as B


@dataclass
class LayerConfig:
    """Quantization of one layer's three matmuls.  The defaults are the benchmark
    configurations' setting: 4-bit codes, Hadamard block 64, 8-bit accumulators over
    tiles of 32, the gradient G rounded stochastically in both backward matmuls and
    everything else to nearest.  The paper's own backward setting (Methodology,
    stochastic-rounding paragraph; Fig. 2 ablation) also rounds the activation
    stochastically in the weight-gradient matmul: `stochastic_act=True`."""
    had_block: int = 64
    bits: int = 4
    acc_bits: int = 8
    s: int = 32
    seed: int = 0
    layer_id: int = 0
    clip_fwd: float = 1.0
    stochastic_grad: bool = True
    stochastic_act: bool = False     # X in dW = X^T G rounded stochastically (the paper's setting)
    need_input_grad: bool = True
    fold_in_matmul: bool = True      # convolution layers: hdqt_conv_bwd where the geometry is taken
    # when set to a dict, every matmul of the layer leaves its operands and results there
    # (X, W, Z in the forward pass; G, dX, dW in the backward pass) for inspection
    capture: Optional[dict] = field(default=None, repr=False, compare=False)

    def params(self, kind: int, step: int = 0) -> B.Params:
        tid = lambda role: 16 * self.layer_id + {"X": 0, "W": 1, "G": 2}[role] + 4 * kind
        NE = B.ROUND_NEAREST
        ST = B.ROUND_STOCHASTIC if self.stochastic_grad else NE
        b = self.bits
        if kind == B.GEMM_FWD:
            A, Bq = B.Operand(b, NE, self.clip_fwd, tid("X")), B.Operand(b, NE, self.clip_fwd, tid("W"))
        elif kind == B.GEMM_BWD_INPUT:
            A, Bq = B.Operand(b, ST, 1.0, tid("G")), B.Operand(b, NE, 1.0, tid("W"))
        else:
            SA = B.ROUND_STOCHASTIC if self.stochastic_act else NE
            A, Bq = B.Operand(b, SA, 1.0, tid("X")), B.Operand(b, ST, 1.0, tid("G"))
        # a fresh random stream every step: the seed advances with the step counter
        return B.Params(had_block=self.had_block, acc_bits=self.acc_bits, s=self.s,
                        seed=self.seed + step, A=A, B=Bq)


class HdqtMatmul(torch.autograd.Function):
    """Z = X W with X [M, K], W [K, N] on the GPU, fp32, contiguous."""

    @staticmethod
    def forward(ctx, X, W, cfg: LayerConfig, step: int):
        # (asked before .contiguous(): a copy made inside forward() does not require grad)
        ctx.want_dx = cfg.need_input_grad and X.requires_grad
        X, W = X.contiguous(), W.contiguous()
        pf = cfg.params(B.GEMM_FWD, step)
        pw = cfg.params(B.GEMM_BWD_WEIGHT, step)
        Z, saved = B.layer_fwd(X, W, pf, pw)
        ctx.save_for_backward(W, saved)
        ctx.cfg, ctx.step, ctx.K = cfg, step, X.shape[1]
        if cfg.capture is not None:
            cfg.capture.update(X=X.detach(), W=W.detach().clone(), Z=Z.detach(), step=step)
        return Z

    @staticmethod
    def backward(ctx, G):
        W, saved = ctx.saved_tensors
        cfg = ctx.cfg
        pi = cfg.params(B.GEMM_BWD_INPUT, ctx.step) if ctx.want_dx else None
        pw = cfg.params(B.GEMM_BWD_WEIGHT, ctx.step)
        G = G.contiguous()
        dX, dW = B.layer_bwd(G, W, saved, ctx.K, pi, pw)
        if cfg.capture is not None:
            cfg.capture.update(G=G.detach(), dX=dX, dW=dW)
        return dX, dW, None, None


class HdqtReluMatmul(torch.autograd.Function):
    """Z = max(pre, 0) W: the rectifier in front of a layer and the layer's matmul as one
    autograd node.  The backward pass returns the gradient of `pre`: the library writes the
    input gradient where the layer's input is positive and zero elsewhere, in the matmul's own
    epilogue (hdqt_layer_bwd_masked), instead of a pass over dX by the framework.  The layer's
    input is kept in fp32 for that (a framework's own rectifier keeps it too)."""

    @staticmethod
    def forward(ctx, pre, W, cfg: LayerConfig, step: int):
        ctx.want_dx = cfg.need_input_grad and pre.requires_grad
        X, W = torch.clamp_min(pre, 0.0).contiguous(), W.contiguous()
        pf = cfg.params(B.GEMM_FWD, step)
        pw = cfg.params(B.GEMM_BWD_WEIGHT, step)
        Z, saved = B.layer_fwd(X, W, pf, pw)
        ctx.save_for_backward(W, saved, X)
        ctx.cfg, ctx.step, ctx.K = cfg, step, X.shape[1]
        if cfg.capture is not None:
            cfg.capture.update(X=X.detach(), W=W.detach().clone(), Z=Z.detach(), step=step)
        return Z

    @staticmethod
    def backward(ctx, G):
        W, saved, X = ctx.saved_tensors
        cfg = ctx.cfg
        pi = cfg.params(B.GEMM_BWD_INPUT, ctx.step) if ctx.want_dx else None
        pw = cfg.params(B.GEMM_BWD_WEIGHT, ctx.step)
        G = G.contiguous()
        dPre, dW = B.layer_bwd(G, W, saved, ctx.K, pi, pw, mask=X if ctx.want_dx else None)
        if cfg.capture is not None:
            cfg.capture.update(G=G.detach(), dX=dPre, dW=dW)
        return dPre, dW, None, None


def _innermost(act: torch.Tensor) -> bool:
    """Whether act [B, C, H, W] has its channels innermost and is of a size that the library's
    transposition is for."""
    if act.is_contiguous() or not act.is_cuda or act.dtype != torch.float32 or act.numel() < 1 << 21:
        return False
    Bn, Cin, H, W = act.shape
    # (the library transposes at most 65535 matrices of 4194240 rows or columns)
    return Bn <= 65535 and max(H * W, Cin) <= 65535 * 64 and act.permute(0, 2, 3, 1).is_contiguous()


def _planes(act: torch.Tensor) -> torch.Tensor:
    """act [B, C, H, W] contiguous.  What comes out of a layer and the normalisation behind it has its
    channels innermost; the library's transposition turns that faster than a strided copy (40 -> 11 us
    for 128 x 64 x 32 x 32, 10.2 -> 9.4 for 128 x 256 x 8 x 8).  Below 2 M elements a call is host time,
    of which the copy has less (128 x 512 x 4 x 4 6.3 / 9.2)."""
    if not _innermost(act) or act.data_ptr() % 16:
        return act.contiguous()
    Bn, Cin, H, W = act.shape
    return B.transpose(act.permute(0, 2, 3, 1).reshape(Bn, H * W, Cin)).reshape(Bn, Cin, H, W)


def _opaque_call_will_do(t: torch.Tensor) -> bool:
    """Whether a library call may stand for an operation on t: t has memory of its own (a batch of
    gradients has none), and no derivative of the result will be asked for (the library's results
    carry no graph and no tangent)."""
    try:
        t.data_ptr()
    except RuntimeError:
        return False
    return not (torch.is_grad_enabled() and t.requires_grad) and \
        torch.autograd.forward_ad.unpack_dual(t).tangent is None


def _fold(dX: torch.Tensor, shape, kh: int, kw: int, stride: int, ph: int, pw: int) -> torch.Tensor:
    """The gradient of an im2col matrix folded back onto the activation of `shape`.  The library's
    kernel has channels as lanes; for fewer than 32 of them PyTorch's fold is the faster one (both
    add an element's terms in the same order)."""
    Bn, Cin, H, W = shape
    if Cin >= 32 and _opaque_call_will_do(dX):
        dX = dX.contiguous()
        if dX.data_ptr() % 16:           # a part of another tensor; the library takes whole 16-byte units
            dX = dX.clone()
        return B.col2im(dX, shape, kh, kw, stride, ph, pw)
    return torch.nn.functional.fold(dX.reshape(Bn, -1, Cin * kh * kw).transpose(1, 2), output_size=(H, W),
                                    kernel_size=(kh, kw), padding=(ph, pw), stride=stride)


def _as_activation(dAct: torch.Tensor, innermost: bool) -> torch.Tensor:
    """The gradient of an activation in the activation's layout.  The kernels write channel planes; behind a
    normalisation everything else has its channels innermost, and PyTorch's elementwise kernels take
    three times as long over two layouts as over one (the rectifier's backward pass at 128 x 64 x 32 x 32
    55 against 16 us, the transposition 12; at 128 x 256 x 8 x 8 17, 5 and 7).  The gradient's values are the same
    bit for bit; what PyTorch adds up behind it (a bias over that activation, say) it may add in another order, as
    behind a gradient of its own in that layout.  For the moment of the transposition there are two of them."""
    if not innermost or dAct.data_ptr() % 16 or not dAct.is_contiguous():
        return dAct
    Bn, Cin, H, W = dAct.shape
    return B.transpose(dAct.reshape(Bn, Cin, H * W)).reshape(Bn, H, W, Cin).permute(0, 3, 1, 2)


_FOLD_REFUSED = set()        # products hdqt_conv_bwd did not take, by everything that this depends on


class HdqtConvMatmul(torch.autograd.Function):
    """Z = im2col(act) W for a stride-1, same-size convolution, without forming im2col(act):
    the forward call reads the activation (hdqt_conv_fwd).  The backward pass returns the
    gradient of the activation: the library's gradient of the im2col matrix, folded back by
    hdqt_col2im where the matmul does not fold it itself."""

    @staticmethod
    def forward(ctx, act, W, cfg: LayerConfig, step: int, kh: int, kw: int):
        ctx.want_dx = cfg.need_input_grad and act.requires_grad
        ctx.innermost = _innermost(act)
        act, W = _planes(act), W.contiguous()
        pf = cfg.params(B.GEMM_FWD, step)
        pw = cfg.params(B.GEMM_BWD_WEIGHT, step)
        Z, saved = B.conv_fwd(act, kh, kw, W, pf, pw)
        ctx.save_for_backward(W, saved)
        ctx.cfg, ctx.step, ctx.shape, ctx.window = cfg, step, tuple(act.shape), (kh, kw)
        if cfg.capture is not None:
            cfg.capture.update(act=act.detach(), W=W.detach().clone(), Z=Z.detach(), step=step)
        return Z

    @staticmethod
    def backward(ctx, G):
        W, saved = ctx.saved_tensors
        cfg = ctx.cfg
        Bn, Cin, H, Wd = ctx.shape
        kh, kw = ctx.window
        pi = cfg.params(B.GEMM_BWD_INPUT, ctx.step) if ctx.want_dx else None
        pw = cfg.params(B.GEMM_BWD_WEIGHT, ctx.step)
        G = G.contiguous()
        dAct = dXcol = None
        key = pi and (ctx.shape, kh, kw, W.shape[1], pi.A.b, pi.B.b, pi.acc_bits, pi.s)
        if pi is not None and cfg.fold_in_matmul and key not in _FOLD_REFUSED:
            # the input gradient folded onto the activation inside the matmul: the gradient of
            # the im2col matrix is never written
            try:
                dAct, dW = B.conv_bwd(G, W, saved, ctx.shape, kh, kw, pi, pw)
            except B.HdqtError as exc:
                if exc.code != -13:
                    raise
                _FOLD_REFUSED.add(key)
        if dAct is None:
            dXcol, dW = B.layer_bwd(G, W, saved, Cin * kh * kw, pi, pw)
            if dXcol is not None:
                dAct = _fold(dXcol, ctx.shape, kh, kw, 1, (kh - 1) // 2, (kw - 1) // 2)
        if dAct is not None:
            dAct = _as_activation(dAct, ctx.innermost)
        if cfg.capture is not None:
            cfg.capture.update(G=G.detach(), dX=dXcol, dAct=dAct, dW=dW)
        return dAct, dW, None, None, None, None


class Unfold(torch.autograd.Function):
    """act [B, C, H, W] -> its im2col matrix [B*Ho*Wo, C*k*k] by the library's one-launch kernel
    (the layers whose geometry the activation-source kernels do not read directly); the
    backward pass folds the matrix gradient back (hdqt_col2im)."""

    @staticmethod
    def forward(ctx, act, k: int, stride: int, pad: int):
        ctx.geo, ctx.innermost = (tuple(act.shape), k, stride, pad), _innermost(act)
        return B.im2col(_planes(act), k, k, stride, pad, pad)

    @staticmethod
    def backward(ctx, dX):
        shape, k, stride, pad = ctx.geo
        dAct = _fold(dX, shape, k, k, stride, pad, pad)
        if ctx.innermost and _opaque_call_will_do(dAct):
            dAct = _as_activation(dAct, True)
        return dAct, None, None, None


class CrossEntropy(torch.autograd.Function):
    """Softmax cross entropy of the classifier X W + bias (hdqt_xent_fwd / hdqt_xent_bwd): the logits are not kept
    between the passes, and formed in pieces of the classes (of 128 MB, or 1024 classes).  X [M, K], W [K, N], both fp32 or bfloat16, target int64 [M]."""

    @staticmethod
    def forward(ctx, X, W, bias, target, ignore_index: int, reduction: str):
        loss, saved = B.xent_fwd(X, W, target, bias, ignore_index, reduction)
        ctx.save_for_backward(X, W, bias, target, saved)
        ctx.how = ignore_index, reduction
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        X, W, bias, target, saved = ctx.saved_tensors
        dX, dW, db = B.xent_bwd(dloss.contiguous(), X, W, target, saved, bias, *ctx.how, need=tuple(ctx.needs_input_grad[:3]))
        return dX, dW, db, None, None, None


class GroupNorm(torch.autograd.Function):
    """Group normalisation with an activation, x [images, ..., channels] contiguous (hdqt_groupnorm_fwd /
    hdqt_groupnorm_bwd): x and the groups' statistics are what is kept for the backward pass."""

    @staticmethod
    def forward(ctx, x, weight, bias, groups: int, eps: float, act: str):
        y, saved = B.groupnorm_fwd(x, groups, weight, bias, eps, act)
        ctx.save_for_backward(x, weight, bias, saved)
        ctx.how = groups, act
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, saved = ctx.saved_tensors
        groups, act = ctx.how
        dx, dw, db = B.groupnorm_bwd(dy.contiguous(), x, saved, groups, weight, bias, act, need=tuple(ctx.needs_input_grad[:3]))
        return dx, dw, db, None, None, None


class GroupNormAct(torch.nn.Module):
    """y = act(group norm(x)), act "none", "relu" or "silu", on activations [B, C, H, W] as layers hand them on: what comes
    out of a layer's product has its channels innermost, which is how this reads and leaves them (an
    activation in channel planes is copied first)."""

    def __init__(self, groups: int, channels: int, eps: float = 1e-5, act: str = "none", device=None):
        super().__init__()
        if channels % groups:
            raise ValueError(f"{channels} channels are no whole groups of {groups}")
        self.groups, self.eps, self.act = groups, eps, act
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(channels, device=device))

    def forward(self, x):
        y = GroupNorm.apply(x.permute(0, 2, 3, 1).contiguous(), self.weight, self.bias, self.groups, self.eps, self.act)
        return y.permute(0, 3, 1, 2)


class ClassifierLoss(torch.nn.Module):
    """A linear classifier and its softmax cross entropy in one, for heads that grow with the tasks of class incremental
    training: `classes` of its columns are in use, the weight keeps room for the rest.  forward(x, target) is the
    loss; logits(x), for evaluation, is PyTorch's product."""

    def __init__(self, in_features: int, num_classes: int, bias: bool = True, classes: Optional[int] = None, ignore_index: int = -100,
                 reduction: str = "mean", device=None):
        super().__init__()
        w = torch.empty(in_features, num_classes, device=device)
        torch.nn.init.normal_(w, std=in_features ** -0.5)
        self.weight = torch.nn.Parameter(w)
        self.bias = torch.nn.Parameter(torch.zeros(num_classes, device=device)) if bias else None
        self.classes = num_classes if classes is None else classes
        self.ignore_index, self.reduction = ignore_index, reduction

    def _used(self):
        n = self.classes
        return self.weight[:, :n], None if self.bias is None else self.bias[:n]

    def forward(self, x, target):
        W, b = self._used()
        return CrossEntropy.apply(x.reshape(-1, x.shape[-1]).contiguous(), W, b, target.reshape(-1).contiguous(), self.ignore_index,
                                  self.reduction)

    def logits(self, x):
        W, b = self._used()
        z = x @ W
        return z if b is None else z + b


def clip_gradients(parameters, max_norm: float, norm_type: float = 2.0, eps: float = 1e-6) -> torch.Tensor:
    """The norm of the parameters' gradients together, which are multiplied in place by min(1, max_norm / (norm + eps))
    (hdqt_clip_grad_norm).  The norm stays on the device: nothing waits for it."""
    parameters = [parameters] if isinstance(parameters, torch.Tensor) else list(parameters)
    grads = [p.grad for p in parameters if p.grad is not None]
    if not grads:
        return torch.zeros((), device=parameters[0].device if parameters else None)
    return B.clip_grad_norm(grads, max_norm, norm_type, eps)


def _as_it_is(how: Optional[B.Dropout]) -> Optional[B.Dropout]:
    """A description for the backward pass, whatever the program does with its own until then."""
    return None if how is None else B.Dropout(how.p, how.seed, how.tensor_id, how.step)


class Dropout(torch.autograd.Function):
    """residual + dropout(x) (hdqt_dropout): no mask is kept, the backward pass forms it again.  x contiguous, residual of its
    shape or None, `how` a binding.Dropout."""

    @staticmethod
    def forward(ctx, x, residual, how: B.Dropout):
        # (the step's tensor is kept as a saved one: whoever advances it before the backward pass is told)
        ctx.save_for_backward(how.step)
        ctx.how = _as_it_is(how)
        return B.dropout(x, how, residual)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        _ = ctx.saved_tensors
        dx = B.dropout(dy.contiguous(), ctx.how) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.needs_input_grad[1] else None, None


class LayerNorm(torch.autograd.Function):
    """Layer normalisation of rows, x [..., columns] contiguous (hdqt_layernorm_fwd / hdqt_layernorm_bwd): y, or, with a residual or
    dropout (a binding.Dropout), y and the sum that was normalised, whose gradient past the normalisation is added to its
    own in the same pass.  What is kept is the sum and the rows' statistics."""

    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps: float, how: Optional[B.Dropout]):
        y, total, saved = B.layernorm_fwd(x, weight, bias, eps, residual, how)
        ctx.save_for_backward(total, saved, weight, None if how is None else how.step)
        ctx.how = _as_it_is(how)
        ctx.set_materialize_grads(False)
        return y if total is x else (y, total)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dtotal=None):
        total, saved, weight, _ = ctx.saved_tensors
        need = tuple(ctx.needs_input_grad[:4])
        if dy is None:                               # (nobody asked for y: only the sum's gradient)
            if dtotal is None:
                return (None,) * 6
            dx = dtotal if ctx.how is None or not need[0] else B.dropout(dtotal.contiguous(), ctx.how)
            return dx if need[0] else None, dtotal if need[1] else None, None, None, None, None
        dx, dres, dw, db = B.layernorm_bwd(dy.contiguous(), total, saved, weight, None if dtotal is None else dtotal.contiguous(), ctx.how, need)
        return dx, dres, dw, db, None, None


class LowRank(torch.autograd.Function):
    """base + scale x A B with an adapter for every row (hdqt_adapters_fwd / hdqt_adapters_bwd): x [M, K], base [M, N], A [n, K, r],
    B [n, r, N], ids int64 [M], scale fp32 [n]; all contiguous."""

    @staticmethod
    def forward(ctx, x, base, A, Bm, ids, scale):
        out, saved = B.adapters_fwd(x, A, Bm, ids, scale, base)
        ctx.save_for_backward(x, A, Bm, ids, scale, saved)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, A, Bm, ids, scale, saved = ctx.saved_tensors
        need = tuple(ctx.needs_input_grad[k] for k in (0, 2, 3))
        grads = B.adapters_bwd(dy.contiguous(), x, A, Bm, ids, saved, scale, need=need) if any(need) else (None,) * 3
        return grads[0], dy if ctx.needs_input_grad[1] else None, grads[1], grads[2], None, None


# ids of the layers that are given none, one after the other: above those that a program counts up
_unnamed = itertools.count(1 << 31)


class _Masks:
    """What a layer with dropout draws its masks by: nothing in evaluation, else a stream of its own (`layer_id`; a layer that is given
    none, and a copy of it, has the next that no other such layer has) that moves with every training call, or, where `counter` is set
    (an int64 tensor of one element on the device, which the program advances), with that: a captured step then takes another
    mask at every replay.  Calls of one layer at one value of the counter have one mask.

    A call that the backward pass makes again (activation checkpointing) takes the mask it had.  Which call that is, torch's random state
    on the host says, which checkpointing sets back as torch's own dropout needs it to: every call draws a number of it, and one
    whose number the layer has seen takes the step that it had then (so does one behind a program's own setting back of that state).
    With a counter nothing is drawn: the program advances it behind the backward pass."""

    REMEMBERED = 4096               # calls whose steps are kept

    def __init__(self, p: float, seed: int, layer_id: Optional[int]):
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"a share of {p} cannot be dropped")
        self.p, self.seed, self.counter, self.unnamed = p, seed, None, layer_id is None
        self.layer_id = next(_unnamed) if self.unnamed else layer_id
        self.step = 0

    def __deepcopy__(self, memo):
        other = copy.copy(self)
        other.counter, other._drawn = copy.deepcopy(self.counter, memo), dict(self._drawn)
        if self.unnamed:
            other.layer_id = next(_unnamed)
        return other

    @property
    def step(self) -> int:
        return self._step

    @step.setter
    def step(self, value: int):
        self._step, self._drawn = int(value), {}

    def _step_of_this_call(self) -> int:
        drawn = torch.empty((), dtype=torch.int64, device="cpu").random_().item()
        step = self._drawn.get(drawn)
        if step is None:
            if torch._C._current_graph_task_id() != -1:
                raise RuntimeError("a forward pass of a layer with dropout, made again by the backward pass, under another random state: its mask is "
                                   "not known (checkpoint with preserve_rng_state, or set masks.counter)")
            step = self._drawn[drawn] = self._step
            self._step += 1
            if len(self._drawn) > self.REMEMBERED:
                del self._drawn[next(iter(self._drawn))]
        return step

    def next(self, training: bool) -> Optional[B.Dropout]:
        if not training or self.p == 0.0:
            return None
        step = self._step_of_this_call() if self.counter is None else self._step
        return B.Dropout(self.p, self.seed + step, self.layer_id, self.counter)


class _Masked(torch.nn.Module):
    """A layer with dropout (`masks`): how far its masks have come is in its state, as `step`, so that a run that is taken up again goes on with
    the next.  A state without it leaves the layer's as it is."""

    def _save_to_state_dict(self, destination, prefix, keep_vars):
        super()._save_to_state_dict(destination, prefix, keep_vars)
        if self.masks.p:
            destination[prefix + "step"] = torch.tensor(self.masks.step, device="cpu")

    def _load_from_state_dict(self, state_dict, prefix, *args):
        step = state_dict.pop(prefix + "step", None)
        if step is not None:
            self.masks.step = int(step)
        super()._load_from_state_dict(state_dict, prefix, *args)


class ResidualDropout(_Masked):
    """residual + dropout(x), or dropout(x); `masks.counter` for captured steps."""

    def __init__(self, p: float, seed: int = 0, layer_id: Optional[int] = None):
        super().__init__()
        self.masks = _Masks(p, seed, layer_id)

    def forward(self, x, residual=None):
        how = self.masks.next(self.training)
        if how is None:
            return x if residual is None else residual + x
        return Dropout.apply(x.contiguous(), None if residual is None else residual.contiguous(), how)


class ResidualNorm(_Masked):
    """A residual block's end: forward(x) is the layer normalisation of x; forward(x, residual) that of the sum
    residual + dropout(x), and the sum, for what follows.  One pass over the tensors either way; `masks.counter` for captured
    steps."""

    def __init__(self, columns: int, eps: float = 1e-5, p: float = 0.0, seed: int = 0, layer_id: Optional[int] = None, device=None):
        super().__init__()
        self.eps, self.masks = eps, _Masks(p, seed, layer_id)
        self.weight = torch.nn.Parameter(torch.ones(columns, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(columns, device=device))

    def forward(self, x, residual=None):
        how = self.masks.next(self.training)
        if residual is None:
            y = LayerNorm.apply(x.contiguous(), None, self.weight, self.bias, self.eps, how)
            return y if how is None else y[0]
        return LayerNorm.apply(x.contiguous(), residual.contiguous(), self.weight, self.bias, self.eps, how)


class Adapters(torch.nn.Module):
    """Low-rank adapters beside a projection of `in_features` to `out_features`, one for each task or request: forward(x, base, ids)
    is base + alpha / rank x A_a B_a with a = ids of the row (negative: base alone).  x and base of any leading shape, ids of that
    shape.  A is drawn, B is zero: an adapter starts as nothing."""

    def __init__(self, in_features: int, out_features: int, adapters: int, rank: int, alpha: Optional[float] = None, device=None):
        super().__init__()
        self.A = torch.nn.Parameter(torch.randn(adapters, in_features, rank, device=device) * in_features ** -0.5)
        self.B = torch.nn.Parameter(torch.zeros(adapters, rank, out_features, device=device))
        self.register_buffer("scale", torch.full((adapters,), (rank if alpha is None else alpha) / rank, device=device))

    def _apply(self, fn, recurse=True):
        # (the scales stay in 32 bits, as the kernels take them, whatever type the module is put into)
        scale = self.scale
        super()._apply(fn, recurse)
        if self.scale.dtype != scale.dtype:
            self.scale = scale.to(self.scale.device)
        return self

    def forward(self, x, base, ids):
        out = LowRank.apply(x.reshape(-1, x.shape[-1]).contiguous(), base.reshape(-1, base.shape[-1]).contiguous(), self.A, self.B,
                            ids.reshape(-1).contiguous(), self.scale.float())
        return out.reshape(base.shape)


class HdqtLinear(torch.nn.Module):
    """y = x W + bias with the matmul and its gradients quantized; inputs of any
    leading shape are flattened to [M, K].  `adapters` (an Adapters of the same features): forward(x, ids) adds those of
    the rows beside it, in floating point; ids are then asked for (negative: none)."""

    def __init__(self, in_features: int, out_features: int, bias: bool = True,
                 cfg: Optional[LayerConfig] = None, device=None, relu_input: bool = False, adapters: Optional[Adapters] = None):
        super().__init__()
        self.adapters = adapters
        self.cfg = cfg or LayerConfig()
        self.relu_input = relu_input      # y = max(x, 0) W + bias, the rectifier's backward pass inside the matmul
        w = torch.empty(in_features, out_features, device=device)
        torch.nn.init.kaiming_normal_(w.t(), nonlinearity="relu")     # fan-in = in_features
        self.weight = torch.nn.Parameter(w)
        self.bias = torch.nn.Parameter(torch.zeros(out_features, device=device)) if bias else None
        self.step = 0

    def forward(self, x, ids=None):
        lead = x.shape[:-1]
        if (ids is None) != (self.adapters is None):
            raise ValueError("ids are for a layer with adapters" if self.adapters is None else
                             "a layer with adapters asks for ids, one for each row (negative: none)")
        fn = HdqtReluMatmul if self.relu_input else HdqtMatmul
        z = fn.apply(x.reshape(-1, x.shape[-1]), self.weight, self.cfg, self.step)
        if self.training:
            self.step += 1
        if self.bias is not None:
            z = z + self.bias
        z = z.reshape(*lead, -1)
        if ids is None:
            return z
        return self.adapters(torch.relu(x) if self.relu_input else x, z, ids)


class HdqtConv2d(torch.nn.Module):
    """Convolution as the paper runs it: the activation is unfolded (im2col, column index =
    channel * kh * kw + tap) and the products of the forward and the backward pass are the
    quantized matmuls above.  Stride-1, same-size layers whose geometry the library takes
    never form the unfolded matrix (hdqt_conv_fwd reads the activation, hdqt_conv_bwd folds the
    input gradient back inside the matmul); the others are unfolded by hdqt_im2col and their
    input gradient is folded back by hdqt_col2im."""

    def __init__(self, in_channels: int, out_channels: int, kernel_size: int = 3, padding: int = 1,
                 stride: int = 1, cfg: Optional[LayerConfig] = None, device=None):
        super().__init__()
        self.k, self.pad, self.stride = kernel_size, padding, stride
        self.cfg = cfg or LayerConfig()
        fan_in = in_channels * kernel_size * kernel_size
        w = torch.empty(fan_in, out_channels, device=device)
        torch.nn.init.kaiming_normal_(w.t(), nonlinearity="relu")
        self.weight = torch.nn.Parameter(w)
        self.step = 0
        self.from_activation = True      # read the activation directly where the library takes the geometry
        self._refused = set()            # input shapes it did not take

    def forward(self, x):
        Bn, Cin, H, W = x.shape
        Ho = (H + 2 * self.pad - self.k) // self.stride + 1
        Wo = (W + 2 * self.pad - self.k) // self.stride + 1
        Z = None
        if (self.from_activation and self.stride == 1 and 2 * self.pad == self.k - 1 and self.training
                and tuple(x.shape) not in self._refused):
            try:
                Z = HdqtConvMatmul.apply(x, self.weight, self.cfg, self.step, self.k, self.k)
            except B.HdqtError as exc:
                if exc.code != -13:
                    raise
                self._refused.add(tuple(x.shape))
        if Z is None:
            X = Unfold.apply(x, self.k, self.stride, self.pad)                     # [B*Ho*Wo, C*k*k]
            Z = HdqtMatmul.apply(X, self.weight, self.cfg, self.step)
        if self.training:
            self.step += 1
        return Z.reshape(Bn, Ho * Wo, -1).transpose(1, 2).reshape(Bn, -1, Ho, Wo)
