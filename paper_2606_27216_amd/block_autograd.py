"""``add_norm``, ``attention`` and ``token_logprob`` as autograd's functions (``block_ops``
calls them where a gradient is asked for). Their backward passes are ``add_norm_grad``,
``attention_grad`` and ``token_logprob_grad``, which cannot be differentiated again."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import block_ops as ops
from .train_autograd import _adjacent


def _rows(g):
    """A gradient as the kernels read it: contiguous, or a matrix whose rows are."""
    return g if g.is_contiguous() or (g.dim() == 2 and g.stride(1) == 1 and g.stride(0) >= g.shape[1]) else g.contiguous()


class AddNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, gain, eps, pack):
        results = ops.add_norm(x, residual, gain, eps, pack)
        ctx.save_for_backward(results[0], gain)
        ctx.eps = eps
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*results[2:])
        return results

    @staticmethod
    @once_differentiable
    def backward(ctx, g_h, g_y, *_):
        h, gain = ctx.saved_tensors
        if g_y is None:  # (the norm was not used: the sum's gradient alone)
            return g_h, g_h, None, None, None
        dh, dgain = ops.add_norm_grad(_rows(g_y), h, gain, None if g_h is None else _rows(g_h), ctx.eps)
        return dh, dh, dgain, None, None


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, eps, pack):
        results = ops.add_norm(x, None, gain, eps, pack)[1:]
        ctx.save_for_backward(x, gain)
        ctx.eps = eps
        ctx.mark_non_differentiable(*results[1:])
        return results

    @staticmethod
    @once_differentiable
    def backward(ctx, g_y, *_):
        x, gain = ctx.saved_tensors
        dx, dgain = ops.add_norm_grad(_rows(g_y), x, gain, None, ctx.eps)
        return dx, dgain, None, None


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_starts, k_starts, q_lengths, k_lengths, causal, scale, workspace):
        out, lse = ops.attention(q, k, v, q_starts, k_starts, q_lengths, k_lengths, causal, scale, workspace=workspace)
        ctx.save_for_backward(q, k, v, out, lse, q_starts, k_starts, q_lengths, k_lengths)
        ctx.causal, ctx.scale = causal, scale
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, g, _):
        grads = ops.attention_grad(_adjacent(g), *ctx.saved_tensors, ctx.causal, ctx.scale)
        return (*grads, None, None, None, None, None, None, None)


class TokenLogprob(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, top, scale):
        # (tensors of their own: views of one could not be written in place)
        results = ops._token_logprob(logits, tokens, top, scale, [logits.new_empty(tokens.shape, dtype=torch.float32) for _ in range(3)])
        ctx.save_for_backward(logits, tokens, results[2], results[1])
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*results[2:])
        return results

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logprob, g_entropy, *_):
        logits, tokens, lse, entropy = ctx.saved_tensors
        g_logprob, g_entropy = (None if g is None else g.contiguous() for g in (g_logprob, g_entropy))
        return ops.token_logprob_grad(g_logprob, g_entropy, logits, tokens, lse, entropy, ctx.scale), None, None, None
