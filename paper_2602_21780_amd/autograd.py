"""The trainable operators as differentiable functions of torch: `xsv.norm_rotate` and `xsv.seq_attend` with their gradients.

Same arguments as the functions of `xsv` without outputs and streams: they run on the current stream of the tensors' device, the
gradient on the stream of the forward pass.  Nothing else is computed here.  Gradients are bf16 like the tensors, those of the
norm's weights and biases fp32; there are no second derivatives.  (As with every function of torch: capture a backward pass into a graph
only while no eager graph over the same leaves is alive.)
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import xsv


def _readable(g):
    """A gradient as the library reads it: autograd also hands over expanded ones, any strides and any place in another tensor."""
    fits = g.stride(2) == 1 and g.stride(0) % 8 == 0 and g.stride(1) % 8 == 0 and 64 <= g.stride(1) <= 1 << 24 and g.data_ptr() % 16 == 0
    return g if fits else g.clone(memory_format=torch.contiguous_format)  # (contiguous() gives back what is contiguous, aligned or not)


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, q_bias, k_weight, k_bias, positions, form):
        weights = dict(q_weight=q_weight, q_bias=q_bias, k_weight=k_weight, k_bias=k_bias)
        q_out, k_out = xsv.norm_rotate(q, k, positions=positions, **weights, **form)
        ctx.save_for_backward(q, k, q_weight, q_bias, k_weight, k_bias, positions)
        ctx.form = form
        return q_out if k is None else (q_out, k_out)

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        q, k, q_weight, q_bias, k_weight, k_bias, positions = ctx.saved_tensors
        grads = [_readable(g) for g in grads]
        sums = any(ctx.needs_input_grad[2:6])
        dq, dk, dw = xsv.norm_rotate_grad(grads[0], None if k is None else grads[1], q, k, positions=positions, q_weight=q_weight, q_bias=q_bias,
                                          k_weight=k_weight, k_bias=k_bias, weight_grads=sums, **ctx.form)
        need = ctx.needs_input_grad
        return (dq if need[0] else None, dk if need[1] else None, *[dw[i] if need[2 + i] else None for i in range(4)], None, None)


def norm_rotate(q, k=None, *, norm="layer", eps=1e-5, q_weight=None, q_bias=None, k_weight=None, k_bias=None, positions=None, base=100.0,
                interleaved=False):
    """xsv.norm_rotate, differentiable by q, k, the weights and the biases.  Returns (q_out, k_out); k_out is None without k."""
    form = dict(norm=norm, eps=eps, base=base, interleaved=interleaved)
    out = _NormRotate.apply(q, k, q_weight, q_bias, k_weight, k_bias, positions, form)
    return (out, None) if k is None else out


class _SeqAttend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_begin, k_begin, form):
        out, lse = xsv.seq_attend(q, k, v, q_begin, k_begin, **form)
        ctx.save_for_backward(q, k, v, out, lse, q_begin, k_begin)
        ctx.form = form
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, _):
        q, k, v, out, lse, q_begin, k_begin = ctx.saved_tensors
        grads = xsv.seq_attend_grad(_readable(dout), q, k, v, out, lse, q_begin, k_begin, **ctx.form)
        return (*[g if need else None for g, need in zip(grads, ctx.needs_input_grad)], None, None, None)


def seq_attend(q, k, v, q_begin, k_begin=None, *, longest_q=None, longest_k=None, causal=0, softmax_scale=0.0):
    """xsv.seq_attend, differentiable by q, k and v.  Returns (out, lse); lse takes part in no gradient."""
    form = dict(longest_q=longest_q, longest_k=longest_k, causal=causal, softmax_scale=softmax_scale)
    return _SeqAttend.apply(q, k, v, q_begin, k_begin, form)
