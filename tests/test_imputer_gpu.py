"""The imputer: the operators together under torch's automatic differentiation."""
import numpy as np
import pytest
import torch

import paper_1511_06416_amd as same
from examples.imputer import train_imputer
from paper_1511_06416_amd import evaluate
from paper_1511_06416_amd.imputer import Imputer, cross_attention, dropout
from tests import cross_reference as ref
from workloads import make_workload

pytestmark = pytest.mark.gpu


def test_gradients_flow_through_both():
    """dropout(attention) + residual: the chain of the two references, with
    the bounds of each pass carried through."""
    dt, drop = torch.float16, 0.25
    q_ptr, k_ptr = [0, 5, 45], [0, 9, 100]
    g = torch.Generator().manual_seed(2)
    q, k, v, dy = (torch.randn(n, 2, 32, generator=g).to(dt).cuda() for n in (45, 100, 100, 45))
    for x in (q, k, v):
        x.requires_grad_()
    plan = same.same_cross_create(q_ptr, k_ptr, 2, 2, 32, dt)
    out = cross_attention(plan, q, k, v, plan.new_workspace(backward=True), drop=drop, seed=3, call_id=1)
    y = dropout(out.flatten(1), drop, 3, 2, residual=out.flatten(1))
    y.backward(dy.flatten(1))
    # the gradient that reaches the attention: dy (1 + keep), rounded as torch does (each branch, then the sum)
    keep = ref.dropout_keep(45, 64, drop, 3, 2).view(45, 2, 32)
    d1 = (dy.cpu().double() * keep).to(dt)
    dout = (d1.float() + dy.cpu().float()).to(dt)
    want = ref.attention(q, k, v, q_ptr, k_ptr, 32 ** -0.5, None, drop, 3, 1, dout)
    ref.check("out", out, *want["out"])
    for n, x in (("dq", q), ("dk", k), ("dv", v)):
        ref.check(n, x.grad, *want[n])


def test_dropout_residual_gradient():
    x, r, dy = (torch.randn(33, 40, device="cuda") for _ in range(3))
    x.requires_grad_()
    r.requires_grad_()
    dropout(x, 0.5, 1, 2, residual=r).backward(dy)
    keep = ref.dropout_keep(33, 40, 0.5, 1, 2)
    assert torch.equal(r.grad, dy) and torch.equal(x.grad.cpu().double(), dy.cpu().double() * keep)


def test_learns_held_out_entries():
    """Answers of held-out entries rank them clearly above chance, as the
    sampler's do."""
    auc, _, _ = train_imputer(make_workload(4), 200)
    assert np.isfinite(auc) and auc > 0.6


def test_answers_follow_the_known_entries():
    """Columns whose unknown entries each equal one known entry, a fair coin:
    nothing but the attention can answer.  Trained on some columns, the network
    answers others; with the known entries of another column, or with all of
    them hidden, it knows nothing (AUC 1/2, its deviation over 12,000 entries
    0.005)."""
    pairs, columns = 6, 2000
    g = torch.Generator(device="cuda").manual_seed(3)
    torch.manual_seed(3)
    net = Imputer(2 * pairs, 2).cuda()
    opt = torch.optim.Adam(net.parameters(), lr=3e-3)
    ptr = np.arange(columns + 1) * pairs
    plan = same.same_cross_create(ptr, ptr, net.heads, net.heads, net.head_dim, net.dtype)
    ws = plan.new_workspace(backward=True)
    known = torch.arange(pairs, device="cuda").repeat(columns)

    def logits(states, **kw):
        return net(plan, ws, known + pairs, known, states, **kw)

    def coins():
        return torch.randint(0, 2, (columns * pairs,), generator=g, device="cuda")

    for s in range(200):
        states = coins()
        loss = torch.nn.functional.cross_entropy(logits(states, drop=0.1, seed=1, call_id=s), states)
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
    with torch.no_grad():
        states = coins()
        other = states.view(columns, pairs).roll(1, 0).flatten()
        hidden = torch.zeros(columns * pairs, dtype=torch.bool, device="cuda")

        def score(out):
            return evaluate.auc((out[:, 1] - out[:, 0]).cpu().numpy(), states.cpu().numpy())

        assert score(logits(states)) > 0.95
        assert abs(score(logits(other)) - 0.5) < 0.03
        assert abs(score(logits(states, key_mask=hidden)) - 0.5) < 0.03
