"""``embed`` and ``qk_norm_rope`` as autograd's functions (``train_ops`` calls them where a
gradient is asked for). Their backward passes are ``embed_grad`` and ``qk_norm_rope_grad``,
which cannot be differentiated again."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import train_ops as ops


def _adjacent(g):
    """A gradient as the kernels read it: elements of a head side by side."""
    return g if g.stride(-1) == 1 or g.shape[-1] == 1 else g.contiguous()


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, scale):
        ctx.save_for_backward(tokens)
        ctx.rows, ctx.scale = table.shape[0], scale
        return ops.embed(tokens, table, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        (tokens,) = ctx.saved_tensors
        return None, ops.embed_grad(tokens, g.contiguous(), ctx.rows, ctx.scale), None


class QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved):
        ctx.save_for_backward(q, k, q_gain, k_gain, cos, sin, positions)
        ctx.eps, ctx.interleaved = eps, interleaved
        return ops.qk_norm_rope(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_q, g_k):
        grads = ops.qk_norm_rope_grad(_adjacent(g_q), _adjacent(g_k), *ctx.saved_tensors, ctx.eps, ctx.interleaved)
        return (*grads, None, None, None, None, None)
