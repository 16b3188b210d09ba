"""The policy update's operators as differentiable functions of torch tensors.

Each wraps a forward and a backward call of ``binding``; what the backward call needs (inputs, outputs, statistics) is kept,
logits never are.  Everything is on the current stream of the tensors' device.  Gradients are of first order: the backward calls
leave no history, so differentiating through a gradient raises.
"""
from __future__ import annotations

import torch

from . import binding as B


class _FirstOrder(torch.autograd.Function):
    """Gradients as they are, with a history that ends in an error.  ``sources``: what they were computed from (torch's once_differentiable
    looks at the incoming gradients alone: of ``f(q).sum()`` they need none, and q's part would be left out without a word)."""
    @staticmethod
    def forward(ctx, n, *grads_and_sources):
        return tuple(None if g is None else g.detach() for g in grads_and_sources[:n])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the gradients of qk_norm_rope, packed_attn and linear_logprob are of first order: they cannot be differentiated again")


def _first_order(grads, sources):
    """What a backward method returns: the plain gradients, unless it runs with create_graph."""
    return _FirstOrder.apply(len(grads), *grads, *sources) if torch.is_grad_enabled() else tuple(grads)


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, inv_freq, sections, eps):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, inv_freq)
        ctx.sections, ctx.eps = sections, eps
        return B.rl_qk_norm_rope(q, k, positions, inv_freq, sections, q_weight, k_weight, eps)

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, positions, inv_freq = ctx.saved_tensors
        grads = B.rl_qk_norm_rope_backward(dq_out.contiguous(), dk_out.contiguous(), q, k, positions, inv_freq, ctx.sections, q_weight, k_weight, ctx.eps)
        return (*_first_order(grads, (dq_out, dk_out, q, k, q_weight, k_weight)), None, None, None, None)


class _PackedAttn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_seqlens, scale):
        out, lse = B.rl_packed_attn(q, k, v, cu_seqlens, scale)
        ctx.save_for_backward(q, k, v, out, lse, cu_seqlens)
        ctx.scale = scale
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, cu_seqlens = ctx.saved_tensors
        grads = B.rl_packed_attn_backward(dout.contiguous(), q, k, v, out, lse, cu_seqlens, ctx.scale)
        return (*_first_order(grads, (dout, q, k, v)), None, None)


class _LinearLogprob(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, token_ids, inv_temperature):
        r = B.rl_linear_logprob(hidden, weight, token_ids, inv_temperature)
        ctx.save_for_backward(hidden, weight, token_ids, r["lse"], r["entropy"])
        ctx.inv_temperature = inv_temperature
        ctx.set_materialize_grads(False)
        return r["logprob"], r["entropy"]

    @staticmethod
    def backward(ctx, g_logprob, g_entropy):
        hidden, weight, token_ids, lse, entropy = ctx.saved_tensors
        if g_logprob is None and g_entropy is None:
            return None, None, None, None
        if g_logprob is None:
            g_logprob = torch.zeros_like(lse)
        want = [n for n, needed in zip(("dhidden", "dweight"), ctx.needs_input_grad) if needed]
        grads = B.rl_linear_logprob_backward(hidden, weight, token_ids, lse, g_logprob.contiguous(),
                                             entropy=None if g_entropy is None else entropy,
                                             g_entropy=None if g_entropy is None else g_entropy.contiguous(),
                                             inv_temperature=ctx.inv_temperature, want=want)
        return (*_first_order(grads, (g_logprob, g_entropy, hidden, weight)), None, None)


def qk_norm_rope(q, k, q_weight, k_weight, positions, inv_freq, sections, eps=1e-6):
    """Norms and rotary embedding of all heads of packed tokens, as ``binding.rl_qk_norm_rope``; gradients reach q, k and the
    weights (float32; None: rotation only)."""
    return _QkNormRope.apply(q, k, q_weight, k_weight, positions, inv_freq, tuple(sections), float(eps))


def packed_attn(q, k, v, cu_seqlens, scale):
    """Causal attention of packed sequences, as ``binding.rl_packed_attn``; gradients reach q, k and v."""
    return _PackedAttn.apply(q, k, v, cu_seqlens, float(scale))


def linear_logprob(hidden, weight, token_ids, inv_temperature=1.0):
    """(logprob, entropy) of the tokens under softmax(inv_temperature * hidden @ weight.T), as ``binding.rl_linear_logprob``; gradients
    reach hidden and weight."""
    return _LinearLogprob.apply(hidden, weight, token_ids, float(inv_temperature))
