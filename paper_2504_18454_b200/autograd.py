"""The block operators as functions that torch's autograd can differentiate.

They keep what the C ABI's backward calls ask for and nothing else; with `checkpoint8` the feed-forward block keeps its
input, gate and up in 8 bits (8.25 bits a value), and its backward pass works on the values that those stand for.
They are differentiable once: under create_graph=True their backward raises RuntimeError.
"""
from __future__ import annotations

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


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, *,
              activation: int = block.ACT_SILU, checkpoint8: bool = False) -> torch.Tensor:
    """`block.ffn_forward` with gradients for x and the three weights."""
    return _GatedFfn.apply(x, w_gate, w_up, w_down, activation, checkpoint8, torch.is_grad_enabled())


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, w_q: torch.Tensor, w_k: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False):
    """`block.qk_norm_rope` with gradients for q, k and the two norm weights."""
    return _QkNormRope.apply(q, k, w_q, w_k, cos, sin, positions, eps, interleaved)
