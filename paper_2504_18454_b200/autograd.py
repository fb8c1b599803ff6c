"""The block operators as functions that torch's autograd can differentiate.

They keep what the C ABI's backward calls ask for and nothing else; with `checkpoint8` the feed-forward block keeps its
input, gate and up in 8 bits (8.25 bits a value), the linear operator its input and what goes into its activation, and their
backward passes work on the values that those stand for.
They are differentiable once: under create_graph=True their backward raises RuntimeError.  As with torch's own functions, no
eager graph of the same leaves may be alive while a backward pass is captured (the engine would make the capture wait for that
graph's stream: an error, and no graph).
"""
from __future__ import annotations

from typing import Optional

import torch

from . import block


def _once(what: str) -> None:
    """Their gradients carry no graph.  (torch's once_differentiable would not do: it raises only where the incoming
    gradient needs one itself, and not for a derivative taken by the inputs.)"""
    if torch.is_grad_enabled():
        raise RuntimeError(f"{what} is differentiable once: its gradients carry no graph, so with create_graph=True a second "
                           "derivative would lack its part")


class _GatedFfn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, activation, checkpoint8, recording):
        needs = recording and any(ctx.needs_input_grad)  # (which stays true under no_grad)
        save = (block.SAVE_8BIT if checkpoint8 else block.SAVE_FULL) if needs else block.SAVE_NONE
        y, saved = block.ffn_forward(x, w_gate, w_up, w_down, activation=activation, save=save)
        if needs:
            ctx.activation, ctx.checkpoint8, ctx.dtype = activation, checkpoint8, x.dtype
            kept = (block.act8_pack(x), *saved) if checkpoint8 else (x, *saved)
            flat = [t for a in kept for t in ((a.q, a.exponent) if checkpoint8 else (a,))]
            ctx.save_for_backward(w_gate, w_up, w_down, *flat)
        return y

    @staticmethod
    def backward(ctx, dy):
        _once("gated_ffn")
        w_gate, w_up, w_down, *kept = ctx.saved_tensors
        if ctx.checkpoint8:
            kept = [block.Act8(kept[i], kept[i + 1], ctx.dtype) for i in (0, 2, 4)]
        x, gate, up = kept
        dy = dy if dy.stride(-1) == 1 or dy.shape[-1] == 1 else dy.contiguous()
        dx, *dw = block.ffn_backward(dy, x, w_gate, w_up, w_down, (gate, up), activation=ctx.activation,
                                     need_dx=ctx.needs_input_grad[0])
        return (dx, *dw, None, None, None)


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, w_q, w_k, cos, sin, positions, eps, interleaved):
        ctx.save_for_backward(q, k, w_q, w_k, cos, sin, positions)
        ctx.eps, ctx.interleaved = eps, interleaved
        return block.qk_norm_rope(q, k, w_q, w_k, cos, sin, positions, eps=eps, interleaved=interleaved)

    @staticmethod
    def backward(ctx, dq, dk):
        _once("qk_norm_rope")
        q, k, *rest = ctx.saved_tensors
        dq, dk = (torch.zeros_like(t) if d is None else d if d.stride(-1) == 1 else d.contiguous()
                  for d, t in ((dq, q), (dk, k)))
        grads = block.qk_norm_rope_backward(dq, dk, q, k, *rest, eps=ctx.eps, interleaved=ctx.interleaved)
        return (*grads, None, None, None, None, None)


def _rows(d: torch.Tensor) -> torch.Tensor:
    """An incoming gradient as the C ABI takes it: the last axis contiguous (that of a sum is expanded)."""
    return d if d.stride(-1) == 1 or d.shape[-1] == 1 else d.contiguous()


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, residual, activation, checkpoint8, recording):
        needs = recording and any(ctx.needs_input_grad[:3])  # (the residual's gradient is the incoming one)
        bent = activation != block.ACT_NONE
        save = (block.SAVE_8BIT if checkpoint8 else block.SAVE_FULL) if needs and bent else block.SAVE_NONE
        y, pre = block.linear_forward(x, w, bias, residual, activation=activation, save=save)
        if needs:
            ctx.activation, ctx.dtype, ctx.eight_x, ctx.eight_pre = activation, x.dtype, checkpoint8, checkpoint8 and bent
            kept = [*block.act8_pack(x)[:2]] if checkpoint8 else [x]
            if bent:
                kept += [pre.q, pre.exponent] if checkpoint8 else [pre]
            ctx.save_for_backward(w, *kept)
        return y

    @staticmethod
    def backward(ctx, dy):
        _once("linear")
        dy, need = _rows(dy), ctx.needs_input_grad
        if not any(need[:3]):
            return None, None, None, dy, None, None, None
        w, *kept = ctx.saved_tensors
        x = block.Act8(kept.pop(0), kept.pop(0), ctx.dtype) if ctx.eight_x else kept.pop(0)
        pre = None if not kept else block.Act8(*kept, ctx.dtype) if ctx.eight_pre else kept[0]
        dx, dw, db = block.linear_backward(dy, x, w, pre, activation=ctx.activation, need_dx=need[0], need_dbias=need[2])
        return dx, dw if need[1] else None, db, dy if need[3] else None, None, None, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, residual, eps, recording):
        needs = recording and any(ctx.needs_input_grad)
        y, total, mean, rstd = block.layer_norm_forward(x, w, b, residual, eps=eps, stats=needs)
        ctx.added = residual is not None
        ctx.set_materialize_grads(False)
        if needs:
            ctx.save_for_backward(total, w, mean, rstd)
        return (y, total) if ctx.added else y

    @staticmethod
    def backward(ctx, dy, dtotal=None):
        _once("layer_norm")
        x, w, mean, rstd = ctx.saved_tensors
        dy = torch.zeros_like(x) if dy is None else _rows(dy)
        dx, dw, db = block.layer_norm_backward(dy, x, w, mean, rstd, None if dtotal is None else _rows(dtotal))
        return dx, dw, db, dx if ctx.added else None, None, None


def _leaf_memory(t: torch.Tensor) -> bool:
    """Whether t is a leaf that takes a gradient, or a view of one.  (A leaf may itself be a view, of an arena's buffer, so that
    the base that a view names need not be the leaf: its gradient's way is followed for as long as it goes to one tensor.)"""
    if t.is_leaf or not t.requires_grad:
        return t.requires_grad
    node, further = None, [t.grad_fn]
    while len(further) == 1:
        node, = further
        further = [f for f, _ in node.next_functions if f is not None]
    leaf = getattr(node, "variable", None)
    return leaf is not None and t.numel() > 0 and leaf.untyped_storage().data_ptr() == t.untyped_storage().data_ptr()


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, in_place):
        if in_place and _leaf_memory(logits):
            raise RuntimeError("cross_entropy: the gradient of a leaf's logits cannot take their place, nor that of a view of a leaf")
        loss, lse = block.cross_entropy_forward(logits, targets)
        ctx.in_place = in_place
        ctx.save_for_backward(logits, targets, lse)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        _once("cross_entropy")
        logits, targets, lse = ctx.saved_tensors
        # (detached: the same memory and version, without the logits' own place in the graph)
        out = logits.detach() if ctx.in_place else None
        return block.cross_entropy_backward(_rows(dloss), logits, targets, lse, out=out), None, None


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, *,
              activation: int = block.ACT_SILU, checkpoint8: bool = False) -> torch.Tensor:
    """`block.ffn_forward` with gradients for x and the three weights."""
    return _GatedFfn.apply(x, w_gate, w_up, w_down, activation, checkpoint8, torch.is_grad_enabled())


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False):
    """`block.qk_norm_rope` with gradients for q, k and the two norm weights."""
    return _QkNormRope.apply(q, k, w_q, w_k, cos, sin, positions, eps, interleaved)


def linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, *,
           activation: int = block.ACT_NONE, checkpoint8: bool = False) -> torch.Tensor:
    """`block.linear_forward` with gradients for x, w, bias and residual."""
    return _Linear.apply(x, w, bias, residual, activation, checkpoint8, torch.is_grad_enabled())


def layer_norm(x: torch.Tensor, w: torch.Tensor, b: torch.Tensor, residual: Optional[torch.Tensor] = None, *, eps: float = 1e-5):
    """`block.layer_norm_forward` with gradients for x, w, b and residual: y, or (y, x + residual) where there is a residual."""
    return _LayerNorm.apply(x, w, b, residual, eps, torch.is_grad_enabled())


def cross_entropy(logits: torch.Tensor, targets: torch.Tensor, *, in_place: bool = False) -> torch.Tensor:
    """`block.cross_entropy_forward`'s losses (K, tokens) with a gradient for the logits.  in_place: the backward pass writes the
    gradient over the logits, which nothing may need any more (autograd tells where it does; a product's backward pass does not
    need its result) and which may be neither a leaf nor a view of one."""
    return _CrossEntropy.apply(logits, targets, in_place)
