"""Second-order gradients of the policy update's functions: there are none, and asking for them is an error, not a silent zero.

The library's calls are replaced by stand-ins of the right shapes, which, like the calls, return tensors without history (no GPU)."""
import pytest
import torch

from paper_2512_21450_amd import autograd as F


def like(*xs):
    return tuple(torch.ones_like(x) for x in xs)


def norms(monkeypatch):
    monkeypatch.setattr(F.B, "rl_qk_norm_rope", lambda q, k, *a: like(q, k))
    monkeypatch.setattr(F.B, "rl_qk_norm_rope_backward", lambda dq, dk, q, k, pos, f, s, qw, kw, eps: like(q, k, qw, kw))
    q, k, w = (torch.rand(*s, requires_grad=True) for s in ((3, 2, 64), (3, 1, 64), (64,)))
    return q, sum(t.sum() for t in F.qk_norm_rope(q, k, w, w, None, None, (8, 12, 12)))


def attention(monkeypatch):
    monkeypatch.setattr(F.B, "rl_packed_attn", lambda q, k, v, cu, scale: (torch.ones_like(q), torch.ones(q.shape[1], q.shape[0])))
    monkeypatch.setattr(F.B, "rl_packed_attn_backward", lambda dout, q, k, v, *a: like(q, k, v))
    q, k, v = (torch.rand(3, h, 64, requires_grad=True) for h in (2, 1, 1))
    return q, F.packed_attn(q, k, v, torch.tensor([0, 3], dtype=torch.int32), 0.1).sum()


def logprob(monkeypatch):
    monkeypatch.setattr(F.B, "rl_linear_logprob", lambda h, w, ids, t: {n: torch.ones(h.shape[0]) for n in ("logprob", "lse", "entropy")})
    monkeypatch.setattr(F.B, "rl_linear_logprob_backward", lambda h, w, *a, **kw: like(h, w))
    h, w = (torch.rand(*s, requires_grad=True) for s in ((3, 64), (7, 64)))
    return h, F.linear_logprob(h, w, torch.zeros(3, dtype=torch.int32))[0].sum()


@pytest.mark.parametrize("call", [norms, attention, logprob])
def test_second_order_gradients_are_refused(monkeypatch, call):
    x, loss = call(monkeypatch)
    (g,) = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="first order"):
        (g.square().sum() + x.square().sum()).backward()


@pytest.mark.parametrize("call", [norms, attention, logprob])
def test_through_the_incoming_gradient_too(monkeypatch, call):
    """the gradient with respect to the incoming gradient is a second-order one as well"""
    x, loss = call(monkeypatch)
    u = torch.ones((), requires_grad=True)
    (g,) = torch.autograd.grad(loss, x, grad_outputs=u, create_graph=True)
    with pytest.raises(RuntimeError, match="first order"):
        torch.autograd.grad(g.sum(), u)


@pytest.mark.parametrize("call", [norms, attention, logprob])
@pytest.mark.parametrize("create_graph", [False, True])
def test_first_order_gradients_pass(monkeypatch, call, create_graph):
    x, loss = call(monkeypatch)
    (g,) = torch.autograd.grad(loss, x, create_graph=create_graph)
    assert (g == 1).all() and g.requires_grad == create_graph
    (x.square().sum() + g.detach().sum()).backward()
    assert torch.equal(x.grad, 2 * x.detach())
