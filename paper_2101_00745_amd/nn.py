"""Drop-in PyTorch layer over the SCC C ABI (the paper's third contribution: SCC as a replacement of the
pointwise convolution inside a depthwise-separable block, trainable end to end).

``SCCFunction`` routes autograd through ``scc_forward`` and ``scc_backward`` (or the single-gradient calls when
only one gradient is wanted);
``SCC`` is the module (weight ``[Cout, Cin//cg]``, optional bias).  All SCC arithmetic runs in the HIP kernels;
the bias, which Section 4.2 only mentions among the trainable parameters, is a broadcast add / a sum over
(N, H, W) done with ordinary tensor ops.  Tensors must be CUDA, contiguous NCHW, float32 or bfloat16.

``DWSCCFunction`` / ``DWSCCBlock`` are the whole DW + SCC block (Eq. 2 feeding the SCC of Section 3.1, nothing in
between): the forward is ``scc_dw_forward`` (one fused kernel where the library prefers it), the backward recomputes
the depthwise output, takes ``scc_backward`` on it and hands the result to ``scc_depthwise3x3_backward``.
"""
import math

import torch

from . import scc as _scc


# where a torch lacks one of these, every call goes the general way
_transforms_active = getattr(torch._C, "_are_functorch_transforms_active", lambda: True)
_tracing_state = getattr(torch._C, "_get_tracing_state", lambda: True)


class _FirstOrder(torch.autograd.Function):
    """Gradients, as a function of the tensors they were computed from, that cannot be differentiated."""

    @staticmethod
    def forward(ctx, count, *tensors):
        return tuple(t.detach() for t in tensors[:count])

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("this operator has no second derivative")


def _first_order(grads, *used):
    """What a backward pass returns.  Under create_graph plain results would be constants, and a loss on them would lose its derivative
    without a word; so they are marked, and only differentiating them is an error."""
    if not torch.is_grad_enabled():
        return grads
    there = [g for g in grads if g is not None]
    marked = iter(_FirstOrder.apply(len(there), *there, *used))
    return tuple(None if g is None else next(marked) for g in grads)


class SCCFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, cg, co):
        x = x.contiguous()
        weight = weight.contiguous()
        ctx.save_for_backward(x, weight)
        ctx.cg, ctx.co = int(cg), float(co)
        return _scc.scc_forward(x, weight, ctx.cg, ctx.co)

    @staticmethod
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        dy = dy.contiguous()
        dx = dw = None
        if ctx.needs_input_grad[0] and ctx.needs_input_grad[1]:
            dx, dw = _scc.scc_backward(x, dy, weight, ctx.cg, ctx.co)      # one call, dy and x read once where fused
        elif ctx.needs_input_grad[0]:
            dx = _scc.scc_backward_input(dy, weight, x.shape[1], ctx.cg, ctx.co)
        elif ctx.needs_input_grad[1]:
            dw = _scc.scc_backward_weight(x, dy, ctx.cg, ctx.co)
        if dw is not None:
            dw = dw.to(weight.dtype)                                        # dw comes back as float32
        return (*_first_order((dx, dw), dy, x, weight), None, None)


def scc(x, weight, cg, co, bias=None):
    """Functional form: y = SCC(x; weight) (+ bias per output channel)."""
    y = SCCFunction.apply(x, weight, cg, co)
    if bias is not None:
        y = y + bias.view(1, -1, 1, 1)
    return y


class SCC(torch.nn.Module):
    """Sliding-channel convolution SCC-cg{cg}-co{co} from ``in_channels`` to ``out_channels`` (Section 3.1)."""

    def __init__(self, in_channels, out_channels, cg=2, co=0.5, bias=False, device="cuda", dtype=torch.float32):
        super().__init__()
        L, _, _ = _scc.scc_window_params(in_channels, out_channels, cg, co)   # validates (Cin, Cout, cg, co)
        self.in_channels, self.out_channels, self.cg, self.co = in_channels, out_channels, int(cg), float(co)
        self.weight = torch.nn.Parameter(torch.empty(out_channels, L, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(out_channels, device=device, dtype=dtype)) if bias else None
        self.reset_parameters()

    def reset_parameters(self):
        L = self.weight.shape[1]
        with torch.no_grad():
            self.weight.normal_(0.0, math.sqrt(2.0 / L))     # He: fan-in of a filter is its window length
            if self.bias is not None:
                self.bias.zero_()

    def forward(self, x):
        return scc(x, self.weight, self.cg, self.co, self.bias)

    def extra_repr(self):
        return "%d, %d, cg=%d, co=%g, bias=%s" % (self.in_channels, self.out_channels, self.cg, self.co,
                                                  self.bias is not None)


class DWSCCFunction(torch.autograd.Function):
    """y = SCC(DW3x3(x; kdw); weight).  The depthwise output z is not kept between the passes: the fused forward
    never writes it, and the backward recomputes it (one more depthwise stage, a fraction of the block's traffic)
    instead of holding an activation-sized tensor per block."""

    @staticmethod
    def forward(ctx, x, kdw, weight, cg, co, dw_stride):
        x, kdw, weight = x.contiguous(), kdw.contiguous(), weight.contiguous()
        ctx.save_for_backward(x, kdw, weight)
        ctx.cg, ctx.co, ctx.s = int(cg), float(co), int(dw_stride)
        return _scc.scc_dw_forward(x, kdw, weight, ctx.cg, ctx.co, ctx.s)

    @staticmethod
    def backward(ctx, dy):
        x, kdw, weight = ctx.saved_tensors
        dy = dy.contiguous()
        need_x, need_k, need_w = ctx.needs_input_grad[:3]
        if need_x and need_k and need_w:                                    # the training step: the three stages in one call
            grads = _scc._dw_backward(x, kdw, weight, dy, ctx.cg, ctx.co, ctx.s, True)   # the gradients in the weights' type
            return (*_first_order(grads, dy, x, kdw, weight), None, None, None)
        z = _scc.scc_depthwise3x3_forward(x, kdw, ctx.s)
        dz = dw = None
        if (need_x or need_k) and need_w:
            dz, dw = _scc.scc_backward(z, dy, weight, ctx.cg, ctx.co)
        elif need_x or need_k:
            dz = _scc.scc_backward_input(dy, weight, z.shape[1], ctx.cg, ctx.co)
        elif need_w:
            dw = _scc.scc_backward_weight(z, dy, ctx.cg, ctx.co)
        dx = dk = None
        if dz is not None:
            dx, dk = _scc.scc_depthwise3x3_backward(x, kdw, dz, ctx.s, need_dx=need_x, need_dk=need_k)
        if dw is not None:
            dw = dw.to(weight.dtype)
        if dk is not None:
            dk = dk.to(kdw.dtype)
        return (*_first_order((dx, dk, dw), dy, x, kdw, weight), None, None, None)


def dw_scc(x, kdw, weight, cg, co, dw_stride=1, bias=None):
    """Functional form of the block: y = SCC(DW3x3(x; kdw); weight) (+ bias per output channel).  A plain training call (dense tensors that all
    want gradients, no tracing, no functional transform) is DWSCCFunction in native code; every other one is DWSCCFunction."""
    y = None
    if not (torch.compiler.is_compiling() or _transforms_active() or _tracing_state() is not None):
        y = (_scc._native or _scc._load_native()).dw_block(x, kdw, weight, cg, co, dw_stride)
    if y is None:
        y = DWSCCFunction.apply(x, kdw, weight, cg, co, dw_stride)
    if bias is not None:
        y = y + bias.view(1, -1, 1, 1)
    return y


class DWSCCBlock(torch.nn.Module):
    """Depthwise 3x3 convolution (spatial stride ``stride``, zero padding 1) followed by SCC-cg{cg}-co{co}: the
    paper's replacement of a standard convolution (Sections 2.2 and 3.1), as one trainable module."""

    def __init__(self, in_channels, out_channels, cg=2, co=0.5, stride=1, bias=False, device="cuda", dtype=torch.float32):
        super().__init__()
        L, _, _ = _scc.scc_window_params(in_channels, out_channels, cg, co)
        self.in_channels, self.out_channels, self.cg, self.co, self.stride = in_channels, out_channels, int(cg), float(co), int(stride)
        self.dw_weight = torch.nn.Parameter(torch.empty(in_channels, 3, 3, device=device, dtype=dtype))
        self.weight = torch.nn.Parameter(torch.empty(out_channels, L, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(out_channels, device=device, dtype=dtype)) if bias else None
        self.reset_parameters()

    def reset_parameters(self):
        with torch.no_grad():
            self.dw_weight.normal_(0.0, math.sqrt(2.0 / 9.0))                 # He: nine taps per depthwise filter
            self.weight.normal_(0.0, math.sqrt(2.0 / self.weight.shape[1]))
            if self.bias is not None:
                self.bias.zero_()

    def forward(self, x):
        return dw_scc(x, self.dw_weight, self.weight, self.cg, self.co, self.stride, self.bias)

    def extra_repr(self):
        return "%d, %d, cg=%d, co=%g, stride=%d, bias=%s" % (self.in_channels, self.out_channels, self.cg, self.co,
                                                             self.stride, self.bias is not None)


class GatedSCCFunction(torch.autograd.Function):
    """y = act(SCC(x; weight[0])) * SCC(x; weight[1]).  Neither projection is kept between the passes: the forward never writes them, and the
    backward computes them again."""

    @staticmethod
    def forward(ctx, x, weight, cg, co, act):
        x, weight = x.contiguous(), weight.contiguous()
        ctx.save_for_backward(x, weight)
        ctx.cg, ctx.co, ctx.act = int(cg), float(co), act
        return _scc.scc_gated_forward(x, weight, ctx.cg, ctx.co, act=act)

    @staticmethod
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        dx, dw = _scc._gated_backward(x, weight, dy.contiguous(), ctx.cg, ctx.co, ctx.act, True)    # dw in the weights' type
        grads = (dx if ctx.needs_input_grad[0] else None, dw if ctx.needs_input_grad[1] else None)
        return (*_first_order(grads, dy, x, weight), None, None, None)


def gated_scc(x, weight, cg, co, act="silu"):
    """Functional form: y = act(SCC(x; weight[0])) * SCC(x; weight[1]), weight [2, Cout, Cin//cg].  Plain training calls run in native code, as
    dw_scc's do."""
    if not (torch.compiler.is_compiling() or _transforms_active() or _tracing_state() is not None):
        y = (_scc._native or _scc._load_native()).gated_block(x, weight, cg, co, _scc._activation(act))
        if y is not None:
            return y
    return GatedSCCFunction.apply(x, weight, cg, co, act)


class GatedSCC(torch.nn.Module):
    """Gated sliding-channel layer from ``in_channels`` to ``out_channels``: two SCCs of the same windows, the first through an activation
    ("silu" or "gelu"), multiplied."""

    def __init__(self, in_channels, out_channels, cg=2, co=0.5, act="silu", device="cuda", dtype=torch.float32):
        super().__init__()
        L, _, _ = _scc.scc_window_params(in_channels, out_channels, cg, co)
        _scc._activation(act)
        self.in_channels, self.out_channels, self.cg, self.co, self.act = in_channels, out_channels, int(cg), float(co), act
        self.weight = torch.nn.Parameter(torch.empty(2, out_channels, L, device=device, dtype=dtype))
        self.reset_parameters()

    def reset_parameters(self):
        with torch.no_grad():
            self.weight.normal_(0.0, math.sqrt(2.0 / self.weight.shape[2]))

    def forward(self, x):
        return gated_scc(x, self.weight, self.cg, self.co, self.act)

    def extra_repr(self):
        return "%d, %d, cg=%d, co=%g, act=%s" % (self.in_channels, self.out_channels, self.cg, self.co, self.act)


class GatedFeedForward(torch.nn.Module):
    """A gated feed-forward block on the channels of [N, channels, H, W]: GatedSCC to ``hidden`` channels, SCC back."""

    def __init__(self, channels, hidden, cg=2, co=0.5, act="silu", device="cuda", dtype=torch.float32):
        super().__init__()
        self.up = GatedSCC(channels, hidden, cg, co, act, device=device, dtype=dtype)
        self.down = SCC(hidden, channels, cg, co, device=device, dtype=dtype)

    def forward(self, x):
        return self.down(self.up(x))


class ResidualNormFunction(torch.autograd.Function):
    """y = norm(x + residual) * weight and h = x + residual.  The backward pass keeps h in float32, x and the residual in bfloat16, where h is rounded."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        x, weight = x.contiguous(), weight.contiguous()
        residual = None if residual is None else residual.contiguous()
        y, h = _scc.scc_norm_forward(x, weight, residual, eps)
        if residual is None:
            ctx.save_for_backward(x, None, weight)
        elif x.dtype == torch.float32:
            ctx.save_for_backward(h, None, weight)
        else:
            ctx.save_for_backward(x, residual, weight)
        ctx.eps = eps
        ctx.set_materialize_grads(False)
        return (y, h) if residual is not None else y

    @staticmethod
    def backward(ctx, dy, dh=None):
        x, residual, weight = ctx.saved_tensors
        if dy is None and dh is None:
            return None, None, None, None
        dh = None if dh is None else dh.contiguous()
        dy = torch.zeros_like(x) if dy is None else dy.contiguous()
        dx, dw = _scc._norm_backward(x, weight, dy, residual, dh, ctx.eps, True)
        need_x, need_r, need_w = ctx.needs_input_grad[:3]
        used = [t for t in (dy, dh, x, residual, weight) if t is not None]
        dx, dw = _first_order((dx if need_x or need_r else None, dw if need_w else None), *used)
        return dx if need_x else None, dx if need_r else None, dw, None


def residual_norm(x, weight, residual=None, eps=1e-6):
    """Functional form: (y, h) with h = x + residual and y = h / sqrt(mean over the channels of h^2 + eps) * weight; without a residual h is x.
    Plain training calls run in native code, as dw_scc's do."""
    if not (torch.compiler.is_compiling() or _transforms_active() or _tracing_state() is not None):
        both = (_scc._native or _scc._load_native()).norm_block(x, weight, residual, eps)
        if both is not None:
            return both
    if residual is None:
        return ResidualNormFunction.apply(x, None, weight, float(eps)), x
    return ResidualNormFunction.apply(x, residual, weight, float(eps))


class ResidualNorm(torch.nn.Module):
    """The norm in front of a feed-forward block, with the addition of the branch before it to the residual stream: (y, h) from (x, residual)."""

    def __init__(self, channels, eps=1e-6, device="cuda", dtype=torch.float32):
        super().__init__()
        self.channels, self.eps = channels, float(eps)
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device, dtype=dtype))

    def forward(self, x, residual=None):
        return residual_norm(x, self.weight, residual, self.eps)

    def extra_repr(self):
        return "%d, eps=%g" % (self.channels, self.eps)


class VocabularyLossFunction(torch.autograd.Function):
    """Cross entropy of the logits x weight^T, which neither pass keeps: the backward pass computes them again, in pieces."""

    @staticmethod
    def forward(ctx, x, weight, target, code, ignore_index):
        x, weight, target = x.contiguous(), weight.contiguous(), target.contiguous()
        loss, lse = _scc.scc_vocabulary_loss(x, weight, target, code, ignore_index)
        ctx.save_for_backward(x, weight, target, lse)
        ctx.code, ctx.ignored = code, ignore_index
        return loss

    @staticmethod
    def backward(ctx, dloss):
        x, weight, target, lse = ctx.saved_tensors
        dx, dw = _scc._vocabulary_gradients(x, weight, target, lse, dloss.contiguous(), _scc._reduction(ctx.code), ctx.ignored, True)
        grads = (dx if ctx.needs_input_grad[0] else None, dw if ctx.needs_input_grad[1] else None)
        return (*_first_order(grads, dloss, x, weight), None, None, None)


def vocabulary_loss(x, weight, target, reduction="mean", ignore_index=-100):
    """Functional form: cross entropy over the vocabulary of logits[n,v,h,w] = sum_c x[n,c,h,w] weight[v,c] at target [N,H,W], float32.
    reduction: "none", "sum" or "mean" (over the targets that are not ignore_index; 0 if there are none).  Plain training calls run in native code, as
    dw_scc's do."""
    if not (torch.compiler.is_compiling() or _transforms_active() or _tracing_state() is not None):
        loss = (_scc._native or _scc._load_native()).vocabulary_block(x, weight, target, _scc._reduction(reduction), ignore_index)
        if loss is not None:
            return loss
    return VocabularyLossFunction.apply(x, weight, target, reduction, int(ignore_index))


class VocabularyLoss(torch.nn.Module):
    """What a model of such blocks ends with in training: the projection of ``channels`` to a vocabulary and the cross entropy, as one."""

    def __init__(self, channels, vocabulary, reduction="mean", ignore_index=-100, device="cuda", dtype=torch.float32):
        super().__init__()
        _scc._reduction(reduction)
        self.channels, self.vocabulary, self.reduction, self.ignore_index = channels, vocabulary, reduction, int(ignore_index)
        self.weight = torch.nn.Parameter(torch.empty(vocabulary, channels, device=device, dtype=dtype))
        self.reset_parameters()

    def reset_parameters(self):
        with torch.no_grad():
            self.weight.normal_(0.0, 1.0 / math.sqrt(self.channels))

    def forward(self, x, target):
        return vocabulary_loss(x, self.weight, target, self.reduction, self.ignore_index)

    def extra_repr(self):
        return "%d, %d, reduction=%s, ignore_index=%d" % (self.channels, self.vocabulary, self.reduction, self.ignore_index)
