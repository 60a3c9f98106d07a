"""Autograd functions and modules over the training operators (ops.py), for models that DistOptim trains: parameters and
their gradients are fp32, activations bf16 or fp32, and what a layer keeps for its backward pass is in 8 bits where the
operator allows it.

    h, y, kept = AddRMSNorm(width)(x, residual)   # kept: y in 8 bits, from the norm's own kernel
    z = CheckpointLinear(width, outs)(y, kept)    # weight gradient from the checkpoint; makes one itself where none is given
    out = attend(q, k, v, causal=True)            # keeps q, k, v, out and the log-sum-exp; recomputes the probabilities

The operators' gradients cannot be differentiated again: second derivatives that need it raise RuntimeError.
"""
from __future__ import annotations

import math
import threading
from typing import Optional, Tuple

import torch

from . import ops


_applied = threading.local()


def _apply(function, *args):
    """The function's apply.  What it keeps is what its backward pass computes with (a log-sum-exp, a norm's factors), and not
    for saved_in_8_bits."""
    outer, _applied.here = getattr(_applied, "here", False), True
    try:
        return function.apply(*args)
    finally:
        _applied.here = outer


class _FirstOrder(torch.autograd.Function):
    """Gradients as they are, as results of the tensors that they depend on: differentiating them raises."""

    @staticmethod
    def forward(ctx, gradients, *tensors):
        return gradients

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("attention, RMS norm and the weight gradient from a checkpoint have no second derivatives")


def _first_order(gradients, *tensors):
    """What the operators give has no graph, so that under create_graph second derivatives would lack it without a word:
    there it is tied to the tensors that it comes from (some may be None)."""
    tensors = [t for t in tensors if t is not None and t.requires_grad]
    return _FirstOrder.apply(gradients, *tensors) if torch.is_grad_enabled() and tensors else gradients


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale, q_lens, kv_lens):
        out, lse = ops.attention(q, k, v, causal=causal, scale=scale, q_lens=q_lens, kv_lens=kv_lens)
        ctx.save_for_backward(q, k, v, out, lse, q_lens, kv_lens)
        ctx.causal, ctx.scale = causal, scale
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, q_lens, kv_lens = ctx.saved_tensors
        grads = ops.attention_backward(dout, q, k, v, out, lse, causal=ctx.causal, scale=ctx.scale, q_lens=q_lens, kv_lens=kv_lens)
        return (*_first_order(grads, dout, q, k, v), None, None, None, None)


def attend(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, scale: Optional[float] = None,
           q_lens: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None) -> torch.Tensor:
    """ops.attention's out, with gradients of q, k and v."""
    return _apply(_Attention, q, k, v, causal, scale, q_lens, kv_lens)


class _AddRMSNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, eps, keep):
        h, y, kept, rstd = ops.add_rms_norm(x, residual, weight, eps, keep=keep)
        ctx.save_for_backward(h, weight, rstd)
        ctx.set_materialize_grads(False)
        if keep:
            ctx.mark_non_differentiable(kept.codes, kept.exponents)
        # without a residual h is x, which an output of its own has to stand for
        return (h if residual is not None else x.view_as(x), y, *(kept[:2] if keep else (None, None)))

    @staticmethod
    def backward(ctx, dh, dy, _codes, _exponents):
        h, weight, rstd = ctx.saved_tensors
        if dy is None:  # nobody used y
            dx, dweight = dh, None
        else:
            dx, dweight = _first_order(ops.add_rms_norm_backward(dy, h, weight, rstd, dh=dh), dy, dh, h, weight)
        return dx, dx if ctx.needs_input_grad[1] else None, dweight, None, None


class AddRMSNorm(torch.nn.Module):
    """h = x + residual; y = h / sqrt(mean(h^2) + eps) * weight.  Gives (h, y, the checkpoint of y), or None in the
    checkpoint's place where the call says that nothing will read it."""

    def __init__(self, width: int, eps: float = 1e-5):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(width))
        self.eps = eps

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, keep: bool = True
                ) -> Tuple[torch.Tensor, torch.Tensor, Optional[ops.Checkpoint]]:
        h, y, codes, exponents = _apply(_AddRMSNorm, x, residual, self.weight, self.eps, keep)
        return h, y, ops.Checkpoint(codes, exponents, self.weight.numel()) if keep else None


class _CheckpointLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, kept, keep):
        rows = x.reshape(-1, x.shape[-1])
        w = weight.to(x.dtype)
        out = rows @ w.t() if bias is None else torch.addmm(bias.to(x.dtype), rows, w.t())
        if not keep:
            kept = ops.Checkpoint(None, None, x.shape[-1])
        elif kept is None:
            kept = ops.checkpoint_encode(rows)
        source = x.new_empty(0)  # of the same inputs as out: what the weight's gradient is tied to, in the place of x
        ctx.save_for_backward(kept.codes, kept.exponents, weight, source)
        ctx.set_materialize_grads(False)
        ctx.cols, ctx.has_bias, ctx.shape = kept.cols, bias is not None, x.shape
        return out.view(*x.shape[:-1], weight.shape[0]), source

    @staticmethod
    def backward(ctx, dout, _source):
        codes, exponents, weight, source = ctx.saved_tensors
        rows = dout.reshape(-1, dout.shape[-1])
        dx = (rows @ weight.to(rows.dtype)).view(ctx.shape) if ctx.needs_input_grad[0] else None
        dw = None
        if ctx.needs_input_grad[1]:
            dw, = _first_order((ops.checkpoint_weight_grad(rows, ops.Checkpoint(codes, exponents, ctx.cols)),), rows, source)
        db = rows.sum(0, dtype=torch.float32) if ctx.has_bias and ctx.needs_input_grad[2] else None
        return dx, dw, db, None, None


class CheckpointLinear(torch.nn.Module):
    """A linear layer that keeps its input in 8 bits for the backward pass: a quarter (fp32) or half (bf16) of the memory.
    Products with the weight are torch's, in the input's type; the weight's gradient is fp32, from the checkpoint."""

    def __init__(self, ins: int, outs: int, bias: bool = True):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(outs, ins))
        self.bias = torch.nn.Parameter(torch.zeros(outs)) if bias else None
        torch.nn.init.uniform_(self.weight, -1 / math.sqrt(ins), 1 / math.sqrt(ins))

    def forward(self, x: torch.Tensor, kept: Optional[ops.Checkpoint] = None) -> torch.Tensor:
        """kept: the checkpoint of x, where it is there already."""
        # a checkpoint is for the weight's gradient alone
        return _apply(_CheckpointLinear, x, self.weight, self.bias, kept, torch.is_grad_enabled() and self.weight.requires_grad)[0]


# Nodes of operations whose result holds its inputs' values: views, copies, casts, parts and what joins them.
_SAME_VALUES = {name + "Backward" for name in (
    "T", "Transpose", "Permute", "View", "UnsafeView", "ReshapeAlias", "Unsqueeze", "Squeeze", "Expand", "Repeat", "AsStrided", "Slice", "Select",
    "Index", "IndexSelect", "Split", "SplitWithSizes", "Unbind", "Unfold", "Diagonal", "Alias", "Clone", "ToCopy", "Cat", "Stack")}


def _of_parameters(node) -> bool:
    """Whether a node of the graph gives values of parameters alone."""
    seen, left = {node}, [node]
    while left:
        node = left.pop()
        if hasattr(node, "variable"):
            if not isinstance(node.variable, torch.nn.Parameter):
                return False
            continue
        sources = {n for n, _ in node.next_functions if n is not None}
        if node.name().rstrip("0123456789") not in _SAME_VALUES or not sources:
            return False
        left += sources - seen
        seen |= sources
    return True


class saved_in_8_bits(torch.autograd.graph.saved_tensors_hooks):
    """Within it, what torch's own operations keep for their backward passes is kept as checkpoints: activations (as a GELU's
    input), which are floating tensors on the GPU of at least `least` elements that were computed on the way of a gradient.
    What is left as it is: parameters and other leaves, what holds values of parameters alone (views, casts, parts, joined ones),
    whatever takes no part in the gradient, as statistics, and rows so short that a checkpoint would be no smaller; also what the
    layers of this file keep.  Not for what has to come back exactly, such as a mask in floating
    point, nor for infinities: a group of 32 neighbours that holds one comes back as NaN.

        with saved_in_8_bits():
            z = torch.nn.functional.gelu(u)
    """

    def __init__(self, least: int = 1 << 16):
        def smaller(t):  # a row's last group is filled up, so that narrow rows are not, and columns (norms' factors) 33 bytes a value
            cols = t.shape[-1] if t.dim() else 1
            return -(-cols // ops.GROUP) * (ops.GROUP + 1) < cols * t.element_size()

        def pack(t):
            if (not t.is_cuda or t.dtype not in (torch.bfloat16, torch.float32) or t.numel() < max(least, 1) or not smaller(t)
                    or t.grad_fn is None or _of_parameters(t.grad_fn) or getattr(_applied, "here", False)):
                # not t: an operation that keeps its own output would be held by what it keeps, for ever
                return t.detach(), t._version
            return ops.checkpoint_encode(t.detach()), t.shape, t.dtype

        def unpack(kept):
            if len(kept) == 2:
                t, version = kept
                if t._version != version:  # torch looks no more, once there are hooks
                    raise RuntimeError("a tensor of shape %s that the backward pass needs was changed in place" % (tuple(t.shape),))
                return t
            checkpoint, shape, dtype = kept
            return ops.checkpoint_decode(checkpoint, dtype).view(shape)
        super().__init__(pack, unpack)


class TransformerBlock(torch.nn.Module):
    """Pre-norm transformer block over (x, residual), as one layer of a stack: attention and a feed-forward network, each
    behind a norm that adds the residual on the way.  Gives the block's (output, residual) for the next one's norm."""

    def __init__(self, width: int, heads: int, kv_heads: Optional[int] = None, ffn: Optional[int] = None, causal: bool = True):
        super().__init__()
        self.heads, self.kv_heads, self.causal = heads, kv_heads or heads, causal
        self.head_dim = width // heads
        self.norm1 = AddRMSNorm(width)
        self.qkv = CheckpointLinear(width, (self.heads + 2 * self.kv_heads) * self.head_dim)
        self.proj = CheckpointLinear(width, width)
        self.norm2 = AddRMSNorm(width)
        self.up = CheckpointLinear(width, ffn or 4 * width)
        self.down = CheckpointLinear(ffn or 4 * width, width)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
                lens: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        batch, tokens, width = x.shape
        trained = torch.is_grad_enabled()
        h, y, kept = self.norm1(x, residual, trained and self.qkv.weight.requires_grad)
        q, k, v = self.qkv(y, kept).view(batch, tokens, -1, self.head_dim).split([self.heads, self.kv_heads, self.kv_heads], 2)
        out = attend(q, k, v, causal=self.causal, q_lens=lens, kv_lens=lens)
        h, y, kept = self.norm2(self.proj(out.reshape(batch, tokens, width)), h, trained and self.up.weight.requires_grad)
        u = self.up(y, kept)
        with saved_in_8_bits():
            z = torch.nn.functional.gelu(u)
        return self.down(z), h
