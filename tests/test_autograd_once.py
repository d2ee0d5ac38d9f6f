"""The gradients that the autograd front end hands on are numbers: a second derivative is refused, not wrong."""
import threading

import pytest
import torch


def _fake_default(monkeypatch):
    """A head of one number: loss = h w, so that dloss/dh = w, and d2(loss^2)/dh2 = 2 w^2, of which dh * g alone would give all or nothing."""
    from paper_2512_21450_b200 import autograd

    class Shared:
        turn = threading.RLock()

        def rl_cross_entropy_fwd_bwd(self, H, W, *args, **kw):
            return dict(loss=(H * W).sum().reshape(1), dH=W.clone(), dW=H.clone(), logp=torch.zeros(1))

        def rl_policy_loss_fwd_bwd(self, H, W, *args, **kw):
            return dict(loss=(H * W).sum().reshape(1), dH=W.clone(), dW=H.clone(), logp=torch.zeros(1), entropy=torch.zeros(1),
                        metrics=torch.zeros(8))
    monkeypatch.setattr(autograd, "default_context", lambda device=0: Shared())
    x = torch.zeros(1)
    return (lambda h, w: autograd.fused_cross_entropy(h, w, x)[0], lambda h, w: autograd.fused_grpo_head_loss(h, w, x, x, x, x, None)[0])


def test_first_derivatives_stay(monkeypatch):
    for loss in _fake_default(monkeypatch):
        h, w = torch.tensor([[3.0]], requires_grad=True), torch.tensor([[5.0]], requires_grad=True)
        (2 * loss(h, w)).backward()
        assert h.grad.item() == 10 and w.grad.item() == 6
        for keep in (False, True):
            gh, = torch.autograd.grad(loss(h, w) ** 2, h, create_graph=keep)
            assert gh.item() == 2 * 15 * 5


def test_second_derivatives_are_refused(monkeypatch):
    for loss in _fake_default(monkeypatch):
        h, w = torch.tensor([[3.0]], requires_grad=True), torch.tensor([[5.0]], requires_grad=True)
        # d(loss^2)/dh = 2 loss w; its derivative in w is 2 h w + 2 loss, of which the stored gradient's own derivative would be missing
        gh, = torch.autograd.grad(loss(h, w) ** 2, h, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            gh.sum().backward()
        gh, = torch.autograd.grad(loss(h, w) ** 2, h, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(gh.sum(), w)
