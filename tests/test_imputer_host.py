"""The autograd functions around the operators, with torch's arithmetic in the
operators' place: what reaches them and what comes back."""
import pytest
import torch

import paper_1511_06416_amd.imputer as imputer


@pytest.fixture
def stand_ins(monkeypatch):
    """Linear stand-ins of the operators; yields the gradients' calls."""
    calls = []

    @torch.no_grad()   # the operators write through addresses
    def dropout(x, y, drop, seed, call_id, residual=None):
        y.copy_(2 * x if residual is None else 2 * x + residual)

    @torch.no_grad()
    def forward(plan, q, k, v, out, lse, workspace, **kw):
        out.copy_(q * q)

    @torch.no_grad()
    def backward(plan, q, k, v, out, lse, dout, dq, dk, dv, workspace, **kw):
        calls.append(dout)
        dq.copy_(2 * q * dout)
        dk.zero_()
        dv.zero_()

    monkeypatch.setattr(imputer, "same_dropout", dropout)
    monkeypatch.setattr(imputer, "same_cross_attention", forward)
    monkeypatch.setattr(imputer, "same_cross_attention_backward", backward)
    yield calls


def penalised(y, x):
    """Gradient of a gradient penalty beside another term."""
    g, = torch.autograd.grad((y ** 3).sum(), x, create_graph=True)
    return torch.autograd.grad((g * g).sum() + (x ** 3).sum(), x)[0]


@pytest.mark.parametrize("branch", [False, True])
def test_dropout_has_derivatives_of_every_order(stand_ins, branch):
    x = torch.randn(4, 16, dtype=torch.float64, requires_grad=True)
    zero = torch.zeros_like(x)
    y = imputer.dropout(zero, 0.5, 0, 0, residual=x) if branch else imputer.dropout(x, 0.5, 0, 0)
    c = 1 if branch else 2
    got = penalised(y, x)
    assert torch.allclose(got, penalised(c * x, x)) and bool(got.ne(3 * x ** 2).any())


def test_second_derivatives_of_attention_are_refused(stand_ins):
    """A gradient penalty must not lose its share silently, through dout or
    through q, k and v."""
    x = torch.randn(4, 2, 8, requires_grad=True)
    kv = torch.zeros(3, 2, 8)
    y = imputer.cross_attention(None, x, kv, kv, None)
    with pytest.raises(RuntimeError, match="second derivatives"):
        penalised(y, x)
    y = imputer.cross_attention(None, x, kv, kv, None)
    g, = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        torch.autograd.grad((g * g).sum() + (x ** 3).sum(), x)
    y = imputer.cross_attention(None, x, kv, kv, None)   # the first one as before
    (y * y).sum().backward()
    assert torch.allclose(x.grad, 4 * x.detach() ** 3)


def test_gradients_arrive_aligned(stand_ins):
    """Whatever view of another gradient reaches the attention: the operator
    takes 16-byte addresses and strides of multiples of eight."""
    q, kv = torch.randn(4, 2, 8, requires_grad=True), torch.zeros(3, 2, 8)
    out = imputer.cross_attention(None, q, kv, kv, None)
    three = torch.zeros(3, requires_grad=True)
    w = torch.randn(3 + out.numel())
    (torch.cat([three, out.flatten()]) * w).sum().backward()   # contiguous, 12 bytes into cat's gradient
    (imputer.cross_attention(None, q, kv, kv, None).transpose(0, 2) * torch.randn(8, 2, 4)).sum().backward()
    out = imputer.cross_attention(None, q, kv, kv, None)
    (torch.cat([torch.zeros(4, 2, 3, requires_grad=True), out], dim=2) * torch.randn(4, 2, 11)).sum().backward()
    assert len(stand_ins) == 3
    for dout in stand_ins:
        assert dout.data_ptr() % 16 == 0 and dout.stride(2) == 1 and not any(s % 8 for s in dout.stride()[:2])
    assert torch.equal(stand_ins[0].flatten(), w[3:])
