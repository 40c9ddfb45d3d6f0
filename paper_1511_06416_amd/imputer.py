"""An amortised imputer beside the sampler: a small network that answers a
column's missing entries from the same column's known entries in one pass,
trained with the library's cross attention and dropout.

``cross_attention`` and ``dropout`` are the library's operators with torch's
automatic differentiation around them; ``Imputer`` is one block of them.  Every
pass runs in the library's HIP kernels; the projections are torch's.  Dropout
is linear and has derivatives of every order; differentiating the attention's
gradients raises.
"""
from __future__ import annotations

import torch

from . import same_cross_attention, same_cross_attention_backward, same_dropout


class _CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, plan, workspace, key_mask, scale, drop, seed, call_id):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        same_cross_attention(plan, q, k, v, out, lse, workspace, key_mask=key_mask, scale=scale, drop=drop, seed=seed,
                             call_id=call_id)
        ctx.save_for_backward(q, k, v, out, lse, key_mask)
        ctx.rest = (plan, workspace, scale, drop, seed, call_id)
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, key_mask = ctx.saved_tensors
        plan, workspace, scale, drop, seed, call_id = ctx.rest
        if dout.numel() and dout.stride(-1) != 1 or any(s % 8 for s in dout.stride()[:2]) or dout.data_ptr() % 16:
            dout = dout.clone(memory_format=torch.contiguous_format)  # contiguous() keeps a misaligned view
        return _CrossGradients.apply(q, k, v, dout, plan, workspace, out, lse, key_mask, scale, drop, seed,
                                     call_id) + (None,) * 7


class _CrossGradients(torch.autograd.Function):
    # A function of its own, so that under create_graph its results hang on
    # what they were computed from and a second derivative finds this node.
    @staticmethod
    def forward(ctx, q, k, v, dout, plan, workspace, out, lse, key_mask, scale, drop, seed, call_id):
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        same_cross_attention_backward(plan, q, k, v, out, lse, dout, dq, dk, dv, workspace, key_mask=key_mask,
                                      scale=scale, drop=drop, seed=seed, call_id=call_id)
        return dq, dk, dv

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("cross_attention: second derivatives are not provided")


def cross_attention(plan, q, k, v, workspace, key_mask=None, scale=None, drop=0.0, seed=0, call_id=0):
    """same_cross_attention as a differentiable function.  workspace serves
    both directions (plan.new_workspace(backward=True)) and, like any
    workspace, one stream at a time."""
    return _CrossAttention.apply(q, k, v, plan, workspace, key_mask, scale, drop, seed, call_id)


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, drop, seed, call_id):
        ctx.rest = (drop, seed, call_id, residual is not None)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        same_dropout(x, y, drop, seed, call_id, residual=residual)
        return y

    @staticmethod
    def backward(ctx, dy):
        drop, seed, call_id, with_residual = ctx.rest
        if dy.stride(-1) != 1:
            dy = dy.contiguous()
        return _Dropout.apply(dy, None, drop, seed, call_id), dy if with_residual else None, None, None, None


def dropout(x, drop, seed, call_id, residual=None):
    """same_dropout as a differentiable function of x and residual; the mask is
    made again in the gradient."""
    return _Dropout.apply(x, residual, drop, seed, call_id)


class Imputer(torch.nn.Module):
    """Logits of node states.  A known entry (node, state) is a key, an entry
    to answer (node) a query of its column; one attention with a residual
    branch, then a matrix per node row of a shared embedding."""

    def __init__(self, n_nodes, max_card, heads=4, head_dim=32, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.head_dim, self.dtype, self.max_card = heads, head_dim, dtype, max_card
        width = heads * head_dim
        self.node = torch.nn.Embedding(n_nodes, width)
        self.entry = torch.nn.Embedding(n_nodes * max_card, 2 * width)
        self.out = torch.nn.Linear(width, width)
        self.answer = torch.nn.Embedding(n_nodes, max_card * width)
        self.bias = torch.nn.Embedding(n_nodes, max_card)
        for e in (self.node, self.entry):
            torch.nn.init.normal_(e.weight, std=0.5)
        torch.nn.init.normal_(self.answer.weight, std=width ** -0.5)
        torch.nn.init.zeros_(self.bias.weight)

    def forward(self, plan, workspace, query_nodes, key_nodes, key_states, key_mask=None, drop=0.0, seed=0, call_id=0):
        """query_nodes, key_nodes, key_states: int64, in the plan's token order."""
        shape = (-1, self.heads, self.head_dim)
        q = self.node(query_nodes).to(self.dtype)
        kv = self.entry(key_nodes * self.max_card + key_states).to(self.dtype)
        k, v = kv.chunk(2, dim=1)
        seen = cross_attention(plan, q.view(shape), k.unflatten(1, shape[1:]), v.unflatten(1, shape[1:]), workspace,
                               key_mask=key_mask, drop=drop, seed=seed, call_id=2 * call_id)
        branch = torch.nn.functional.linear(seen.flatten(1), self.out.weight.to(self.dtype),
                                            self.out.bias.to(self.dtype))
        y = dropout(branch, drop, seed, 2 * call_id + 1, residual=seen.flatten(1)).float()
        w = self.answer(query_nodes).unflatten(1, (self.max_card, -1))
        return (w * y[:, None, :]).sum(dim=2) + self.bias(query_nodes)
