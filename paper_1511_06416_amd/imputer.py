"""An amortised imputer beside the sampler: a small network that answers a
column's missing entries from the same column's known entries in one pass,
trained with the library's operators.

``cross_attention``, ``dropout``, ``qk_norm`` and ``log_probs`` are the library's
operators with torch's automatic differentiation around them; ``Imputer`` is one
block of them, and ``Orthogonal`` the optimiser of its matrices.  Every pass
runs in the library's HIP kernels; the projections are torch's.  Dropout is
linear and has derivatives of every order; differentiating the others' gradients
raises.  As with torch's own operators, a backward pass can be captured into a
graph once no eager pass over the same parameters is alive: torch would have it
accumulate on that one's stream.
"""
from __future__ import annotations

import numpy as np
import torch

from . import (NEWTON_SCHULZ, same_cross_attention, same_cross_attention_backward, same_dropout, same_log_probs,
               same_log_probs_backward, same_log_probs_workspace_size, same_orthogonalise,
               same_orthogonalise_workspace_size, same_qk_norm, same_qk_norm_backward, same_qk_norm_workspace_size)


def _aligned(g):
    """A gradient of heads as the operators take it: contiguous() would keep a
    misaligned view."""
    if g.numel() and (g.stride(-1) != 1 or any(s % 8 for s in g.stride()[:2]) or g.data_ptr() % 16):
        return g.clone(memory_format=torch.contiguous_format)
    return g


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
        return _CrossGradients.apply(q, k, v, _aligned(dout), plan, workspace, out, lse, key_mask, scale, drop, seed,
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


class _QkNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, q_positions, k_positions, angles, eps):
        if angles is not None:   # the backward pass turns by what the forward pass did, whatever becomes of the caller's
            angles = np.array(angles, dtype=np.float64)
        q_out, k_out = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        same_qk_norm(q, k, q_out, k_out, q_weight=q_weight, k_weight=k_weight, q_positions=q_positions,
                     k_positions=k_positions, angles=angles, eps=eps)
        ctx.save_for_backward(q, k, q_weight, k_weight, q_positions, k_positions)
        ctx.rest = (angles, eps)
        return q_out, k_out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, q_positions, k_positions = ctx.saved_tensors
        grads = _QkNormGradients.apply(q, k, q_weight, k_weight, _aligned(dq_out), _aligned(dk_out), q_positions,
                                       k_positions, *ctx.rest, *ctx.needs_input_grad[2:4])
        return grads + (None,) * 4


class _QkNormGradients(torch.autograd.Function):
    # as _CrossGradients: a second derivative finds this node
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, dq_out, dk_out, q_positions, k_positions, angles, eps, for_q, for_k):
        dq, dk = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        dq_weight = torch.empty_like(q_weight) if for_q else None
        dk_weight = torch.empty_like(k_weight) if for_k else None
        workspace = None
        if for_q or for_k:
            need = same_qk_norm_workspace_size(q.shape[2], q.shape[0], q.shape[1], k.shape[0], k.shape[1])
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
        same_qk_norm_backward(q, k, dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace, q_weight=q_weight,
                              k_weight=k_weight, q_positions=q_positions, k_positions=k_positions, angles=angles,
                              eps=eps)
        return dq, dk, dq_weight, dk_weight

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("qk_norm: second derivatives are not provided")


def qk_norm(q, k, q_weight=None, k_weight=None, q_positions=None, k_positions=None, angles=None, eps=1e-6):
    """same_qk_norm as a differentiable function of q, k and the weights."""
    return _QkNorm.apply(q, k, q_weight, k_weight, q_positions, k_positions, angles, eps)


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, counts, n_top):
        rows, cols = logits.shape
        new = {"device": logits.device, "dtype": torch.float32}
        out = None if targets is None else torch.empty(rows, **new)
        sums, entropy = torch.empty(rows, 2, **new), torch.empty(rows, **new)
        ids = top = None
        if n_top:
            ids = torch.empty(rows, n_top, dtype=torch.int32, device=logits.device)
            top = torch.empty(rows, n_top, **new)
        workspace = torch.empty(max(same_log_probs_workspace_size(rows, cols, n_top), 1), dtype=torch.uint8,
                                device=logits.device)
        same_log_probs(logits, targets, out, workspace, counts=counts, sums=sums, entropy=entropy, top_ids=ids,
                       top_log_probs=top)
        ctx.save_for_backward(logits, targets, counts, sums, entropy)
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*(t for t in (ids, top) if t is not None))
        return out, entropy, ids, top

    @staticmethod
    def backward(ctx, d_out, d_entropy, d_ids, d_top):
        logits, targets, counts, sums, entropy = ctx.saved_tensors
        if d_out is None and d_entropy is None:
            return None, None, None, None
        d_out, d_entropy = (None if d is None else d.contiguous() for d in (d_out, d_entropy))
        return _LogProbsGradient.apply(logits, d_out, d_entropy, targets, counts, sums, entropy), None, None, None


class _LogProbsGradient(torch.autograd.Function):
    # as _CrossGradients: a second derivative finds this node
    @staticmethod
    def forward(ctx, logits, d_out, d_entropy, targets, counts, sums, entropy):
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        same_log_probs_backward(logits, targets, sums, dlogits, counts=counts, entropy=entropy, dlog_probs=d_out,
                                dentropy=d_entropy)
        return dlogits

    @staticmethod
    def backward(ctx, grad):
        raise RuntimeError("log_probs: second derivatives are not provided")


def log_probs(logits, targets=None, counts=None, n_top=0):
    """same_log_probs as a differentiable function of logits: the log
    probabilities of targets (int32; None without them), the entropy, and the
    n_top most likely states (int32) with their log probabilities (None with
    n_top = 0).  The latter two carry no gradient."""
    return _LogProbs.apply(logits, targets, counts, n_top)


class Orthogonal(torch.optim.Optimizer):
    """Momentum whose update is orthogonalised, for parameters that are
    matrices: rows x cols, [n][rows][cols], or any shape with `shape` = (rows,
    cols) in their group, which holds one matrix after another.

        m <- momentum m + g,  u = g + momentum m (nesterov) or m
        w <- (1 - lr weight_decay) w - lr sqrt(max(1, rows / cols)) orthogonalise(u)

    Momentum is held in 32 bits whatever the parameter's type; the first step
    creates it and cannot be captured into a graph, later ones can.  u is
    orthogonalised in the parameter's type; of fp16 parameters in 32 bits, as sums
    of gradients pass fp16's range.

    An update has the same size however small u is: a matrix whose gradient is zero
    (a node's that no column of the minibatch asks for) goes on with full steps
    until its momentum falls below eps, some 300 steps after a gradient of norm 1.
    """

    def __init__(self, params, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, coefs=NEWTON_SCHULZ,
                 eps=1e-7, shape=None):
        if lr < 0 or not 0 <= momentum < 1 or weight_decay < 0:
            raise ValueError("lr and weight_decay must not be negative, momentum must lie in [0, 1)")
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay,
                                      coefs=coefs, eps=eps, shape=shape))
        for group in self.param_groups:
            for p in group["params"]:
                self._shape(p, group)

    @staticmethod
    def _shape(p, group):
        shape = group["shape"]
        if shape is not None:
            rows, cols = shape
            if rows < 1 or cols < 1:
                raise ValueError("shape must be a matrix's, got %s" % (tuple(shape),))
            if p.numel() % (rows * cols):
                raise ValueError("a parameter of shape %s holds no whole matrices of %d x %d"
                                 % (tuple(p.shape), rows, cols))
            return (p.numel() // (rows * cols), rows, cols)
        if p.dim() not in (2, 3):
            raise ValueError("a parameter of shape %s is neither a matrix nor a row of them" % (tuple(p.shape),))
        return (1, *p.shape) if p.dim() == 2 else tuple(p.shape)

    @staticmethod
    def _wide(p):
        return torch.promote_types(p.dtype, torch.float32)

    def load_state_dict(self, state_dict):
        """As torch's, which would give the momentum its parameter's type."""
        super().load_state_dict(state_dict)
        saved = [i for group in state_dict["param_groups"] for i in group["params"]]
        params = [p for group in self.param_groups for p in group["params"]]
        for i, p in zip(saved, params):
            if "momentum" in state_dict["state"].get(i, ()):
                self.state[p]["momentum"] = state_dict["state"][i]["momentum"].to(p.device, self._wide(p), copy=True)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            lr, momentum = group["lr"], group["momentum"]
            for p in group["params"]:
                if p.grad is None or not p.numel():
                    continue
                shape = self._shape(p, group)
                state = self.state[p]
                if "momentum" not in state:
                    if p.is_cuda and torch.cuda.is_current_stream_capturing():   # every replay would clear it
                        raise RuntimeError("Orthogonal: the first step creates the momentum; take it before the capture")
                    state["momentum"] = torch.zeros_like(p, dtype=self._wide(p), memory_format=torch.contiguous_format)
                m = state["momentum"].mul_(momentum).add_(p.grad)
                u = p.grad.add(m, alpha=momentum) if group["nesterov"] else m
                u = u.to(torch.float32 if p.dtype is torch.float16 else p.dtype).contiguous().view(shape)
                out = torch.empty_like(u)
                workspace = torch.empty(max(same_orthogonalise_workspace_size(*shape, u.dtype), 1), dtype=torch.uint8,
                                        device=u.device)
                same_orthogonalise(u, out, workspace, coefs=group["coefs"], eps=group["eps"],
                                   scale=max(1.0, shape[1] / shape[2]) ** 0.5)
                if group["weight_decay"]:
                    p.mul_(1.0 - lr * group["weight_decay"])
                p.add_(out.view(p.shape), alpha=-lr)
        return loss


class Imputer(torch.nn.Module):
    """Logits of node states.  A known entry (node, state) is a key, an entry
    to answer (node) a query of its column; one attention with a residual
    branch, then a matrix per node row of a shared embedding.  With norm the
    heads of queries and keys are normed before the attention and, with rot_dim,
    turned by the positions that forward is given, for instance an entry's
    column where a segment holds several."""

    def __init__(self, n_nodes, max_card, heads=4, head_dim=32, dtype=torch.bfloat16, norm=False, rot_dim=0):
        super().__init__()
        if rot_dim and not norm:
            raise ValueError("rot_dim needs norm")
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
        self.norm = norm
        self.angles = 10_000.0 ** (-2.0 * np.arange(rot_dim // 2) / max(rot_dim, 1)) if rot_dim else None
        if norm:
            self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(head_dim)) for _ in range(2))

    def forward(self, plan, workspace, query_nodes, key_nodes, key_states, key_mask=None, drop=0.0, seed=0, call_id=0,
                query_positions=None, key_positions=None):
        """query_nodes, key_nodes, key_states: int64, in the plan's token order; positions (with rot_dim): int32."""
        shape = (-1, self.heads, self.head_dim)
        q = self.node(query_nodes).to(self.dtype).view(shape)
        kv = self.entry(key_nodes * self.max_card + key_states).to(self.dtype)
        k, v = (x.unflatten(1, shape[1:]) for x in kv.chunk(2, dim=1))
        if self.norm:
            q, k = qk_norm(q, k, self.q_weight, self.k_weight, query_positions, key_positions, self.angles)
        seen = cross_attention(plan, q, k, v, workspace, key_mask=key_mask, drop=drop, seed=seed, call_id=2 * call_id)
        branch = torch.nn.functional.linear(seen.flatten(1), self.out.weight.to(self.dtype),
                                            self.out.bias.to(self.dtype))
        y = dropout(branch, drop, seed, 2 * call_id + 1, residual=seen.flatten(1)).float()
        w = self.answer(query_nodes).unflatten(1, (self.max_card, -1))
        return (w * y[:, None, :]).sum(dim=2) + self.bias(query_nodes)

    def optimisers(self, lr=0.02, other_lr=3e-3):
        """Orthogonalised updates for the output matrix and the nodes' answer
        matrices, Adam for the embeddings, weights and biases."""
        matrices = [dict(params=[self.out.weight]),
                    dict(params=[self.answer.weight], shape=(self.max_card, self.heads * self.head_dim))]
        taken = {id(self.out.weight), id(self.answer.weight)}
        rest = [p for p in self.parameters() if id(p) not in taken]
        return Orthogonal(matrices, lr=lr), torch.optim.Adam(rest, lr=other_lr)
