"""Autograd functions and modules over the training operators (ops.py), for models that DistOptim trains: parameters and
their gradients are fp32, activations bf16 or fp32, and what a layer keeps for its backward pass is in 8 bits where the
operator allows it.

    h, y, kept = AddRMSNorm(width)(x, residual)   # kept: y in 8 bits, from the norm's own kernel
    z = CheckpointLinear(width, outs)(y, kept)    # weight gradient from the checkpoint; makes one itself where none is given
    out = attend(q, k, v, causal=True)            # keeps q, k, v, out and the log-sum-exp; recomputes the probabilities
    h, last = recur(x, gate, state)               # keeps x, the gates and every 256th state; recomputes the others
    y = ExpertLinear(experts, ins, outs)(x, ends) # keeps x; rows sorted by expert

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
        raise RuntimeError("attention, RMS norm, the recurrence, products by expert and the weight gradient from a checkpoint have no second "
                           "derivatives")


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


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, state, lens, keep):
        h, last, kept = ops.recurrence(x, gate, state, lens, keep=keep)
        # nothing is computed from the state: where it has a gradient, that is tied to it
        ctx.save_for_backward(x, gate, kept, lens, state if ctx.needs_input_grad[2] else None)
        ctx.set_materialize_grads(False)
        return h, last

    @staticmethod
    def backward(ctx, dh, dlast):
        x, gate, kept, lens, state = ctx.saved_tensors
        if dh is None and dlast is None:
            return None, None, None, None, None
        given = dh, dlast
        if dh is None:
            dh = torch.zeros_like(x)
        grads = ops.recurrence_backward(dh, x, gate, kept, lens, None if dlast is None else dlast.contiguous())
        dx, dgate, dstate = _first_order(grads, *given, x, gate, state)
        return dx, dgate, dstate if ctx.needs_input_grad[2] else None, None, None


def recur(x: torch.Tensor, gate: torch.Tensor, state: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None
          ) -> Tuple[torch.Tensor, torch.Tensor]:
    """ops.recurrence's h and last, with gradients of x, the gates and the state."""
    keep = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, gate, state))
    return _apply(_Recurrence, x, gate, state, lens, keep)


class _ExpertLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, ends):
        ctx.save_for_backward(x, weight, ends)
        return ops.expert_linear(x, weight.to(x.dtype), ends)

    @staticmethod
    def backward(ctx, dy):
        x, weight, ends = ctx.saved_tensors
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx, = _first_order((ops.expert_input_grad(dy, weight.to(dy.dtype), ends),), dy, weight)
        if ctx.needs_input_grad[1]:
            dw, = _first_order((ops.expert_weight_grad(dy, x, ends).to(weight.dtype),), dy, x)
        return dx, dw, None


class ExpertLinear(torch.nn.Module):
    """A linear layer for each of several experts, without biases: rows [M, ins] sorted by expert, expert e's up to row ends[e]; rows
    behind the last one's give 0.  Parameters and their gradients are fp32, products in the rows' type."""

    def __init__(self, experts: int, ins: int, outs: int):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(experts, outs, ins))
        torch.nn.init.uniform_(self.weight, -1 / math.sqrt(ins), 1 / math.sqrt(ins))

    def forward(self, x: torch.Tensor, ends: torch.Tensor) -> torch.Tensor:
        return _apply(_ExpertLinear, x, self.weight, ends)


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


class _Spread(torch.autograd.Function):
    """Rows [M, width], each to `top` places: out[place[m, i]] = rows[m].  Gradients are added over the places in their order."""

    @staticmethod
    def forward(ctx, rows, place, source):
        ctx.save_for_backward(place, source)
        return rows[source]

    @staticmethod
    def backward(ctx, dout):
        place, source = ctx.saved_tensors
        return _Gather.apply(dout, place, source).sum(1), None, None


class _Gather(torch.autograd.Function):
    """out[m, i] = rows[place[m, i]], with every row in one place."""

    @staticmethod
    def forward(ctx, rows, place, source):
        ctx.save_for_backward(place, source)
        return rows[place]

    @staticmethod
    def backward(ctx, dout):
        place, source = ctx.saved_tensors
        flat = dout.flatten(0, 1)
        order = torch.empty_like(source).scatter_(0, place.flatten(), torch.arange(source.numel(), device=source.device))
        return flat[order], None, None


class Experts(torch.nn.Module):
    """Feed-forward layer of several experts: a router sends each token to `top` of them, whose results are added with the router's
    weights (a softmax over the chosen ones).  Tokens behind the sequences' lengths go to none, and give 0."""

    def __init__(self, width: int, ffn: int, experts: int, top: int = 2):
        super().__init__()
        if not 1 <= top <= experts:
            raise ValueError("top %d of %d experts" % (top, experts))
        self.experts, self.top = experts, top
        self.router = torch.nn.Parameter(torch.empty(experts, width))
        torch.nn.init.uniform_(self.router, -1 / math.sqrt(width), 1 / math.sqrt(width))
        self.up = ExpertLinear(experts, width, ffn)
        self.down = ExpertLinear(experts, ffn, width)

    def forward(self, y: torch.Tensor, lens: Optional[torch.Tensor] = None) -> torch.Tensor:
        batch, tokens, width = y.shape
        rows = y.reshape(-1, width)
        if lens is not None:
            valid = (torch.arange(tokens, device=y.device) < lens.view(-1, 1)).view(-1, 1)
            rows = torch.where(valid, rows, 0)  # what stands behind the lengths may be anything: the router is not to see it
        # chosen in fp32, whatever the activations' type: a rounding must not send a token elsewhere
        scores, chosen = (rows.float() @ self.router.t()).topk(self.top, -1)
        share = torch.softmax(scores, -1)
        if lens is not None:
            chosen = torch.where(valid, chosen, self.experts)
            share = torch.where(valid, share, 0)  # nor what the incoming gradient holds there: it would reach the router through the softmax
        sorted_, order = chosen.flatten().sort(stable=True)
        ends = torch.searchsorted(sorted_, torch.arange(self.experts, device=y.device), right=True).to(torch.int32)
        place = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=y.device)).view(-1, self.top)
        u = self.up(_Spread.apply(rows, place, order // self.top), ends)
        with saved_in_8_bits():
            z = torch.nn.functional.gelu(u)
        z = _Gather.apply(self.down(z, ends), place, order // self.top)
        return (z * share.unsqueeze(2).to(z.dtype)).sum(1).view(y.shape)


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


class RecurrentBlock(torch.nn.Module):
    """Pre-norm block over (x, residual) as TransformerBlock, with a gated linear recurrence in the place of attention, whose result is
    gated by the token, and a feed-forward network or, with `experts`, several of them.  Gives the block's (output, residual)."""

    def __init__(self, width: int, ffn: Optional[int] = None, experts: int = 0, top: int = 2):
        super().__init__()
        self.norm1 = AddRMSNorm(width)
        self.into = CheckpointLinear(width, 3 * width)
        self.proj = CheckpointLinear(width, width)
        self.norm2 = AddRMSNorm(width)
        self.experts = Experts(width, ffn or 4 * width, experts, top) if experts else None
        if not experts:
            self.up = CheckpointLinear(width, ffn or 4 * width)
            self.down = CheckpointLinear(ffn or 4 * width, width)
        with torch.no_grad():  # memories of some steps to some hundred
            self.into.bias[width:2 * width] = torch.linspace(1, 6, width)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None,
                state: Optional[torch.Tensor] = None):
        """With a state (fp32 [batch, width], zeros at a sequence's start) also the state behind these tokens, for a call on the next."""
        width = x.shape[-1]
        trained = torch.is_grad_enabled()
        h, y, kept = self.norm1(x, residual, trained and self.into.weight.requires_grad)
        v, gate, open_ = self.into(y, kept).split(width, 2)
        s, last = recur(v, gate, state, lens)
        h, y, kept = self.norm2(self.proj(s * torch.nn.functional.silu(open_)), h,
                                trained and self.experts is None and self.up.weight.requires_grad)
        if self.experts is not None:
            out = self.experts(y, lens)
        else:
            u = self.up(y, kept)
            with saved_in_8_bits():
                z = torch.nn.functional.gelu(u)
            out = self.down(z)
        return (out, h) if state is None else (out, h, last)
