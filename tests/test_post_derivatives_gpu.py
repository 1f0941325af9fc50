"""Derivatives that the post-training operators do not have are refused, not left out."""

import pytest
import torch
import torch.autograd.forward_ad as fw

from paper_2608_09703_amd import api as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _norm():
    x, w, b = torch.randn(5, 64, device=DEV), torch.randn(64, device=DEV), torch.randn(64, device=DEV)
    return [x, w, b], lambda x, w, b: D.layer_norm(x, w, b)


def _logp():
    h, W = torch.randn(5, 64, device=DEV), torch.randn(30, 64, device=DEV)
    tokens = torch.arange(5, device=DEV)
    return [h, W], lambda h, W: D.token_logp(h, W, tokens)[0]


def _policy():
    logp, old, adv = (torch.randn(9, device=DEV) for _ in range(3))
    return [logp], lambda logp: D.policy_loss(logp, old, adv)[0]


OPS = [_norm, _logp, _policy]


@pytest.mark.parametrize("make", OPS, ids=lambda f: f.__name__[1:])
@pytest.mark.parametrize("grad", [False, True])
def test_forward_mode_is_refused(make, grad):
    args, f = make()
    want = f(*args)
    with fw.dual_level():
        for i in range(len(args)):
            dual = list(args)
            dual[i] = fw.make_dual(args[i], torch.ones_like(args[i]))
            if grad:
                dual = [x if j == i else x.detach().requires_grad_(True) for j, x in enumerate(dual)]
            with pytest.raises(NotImplementedError):
                f(*dual)
            with torch.no_grad(), pytest.raises(NotImplementedError):
                f(*dual)
        assert torch.equal(f(*args), want)  # other tensors of the level are as before


@pytest.mark.parametrize("make", OPS, ids=lambda f: f.__name__[1:])
def test_forward_mode_over_the_backward_is_refused(make):
    args, f = make()
    leaves = [x.requires_grad_(True) for x in args]
    y = f(*leaves)
    with fw.dual_level():
        g = fw.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises(NotImplementedError):
            torch.autograd.grad(y, leaves, g, retain_graph=True)
        torch.autograd.grad(y, leaves, torch.ones_like(y))


@pytest.mark.parametrize("make", OPS, ids=lambda f: f.__name__[1:])
def test_gradients_of_gradients_are_refused(make):
    args, f = make()
    leaves = [x.requires_grad_(True) for x in args]
    y = f(*leaves)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y.sum(), leaves, create_graph=True)
