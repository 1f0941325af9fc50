"""The clipped policy loss at the ends of its ranges, against the float64 oracle."""

import numpy as np
import pytest
import torch

from oracle import post as P
from paper_2608_09703_amd import api as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


def _np(x):
    return x.detach().double().cpu().numpy()


@pytest.mark.parametrize("N", [1500, 5000, 70000])
@pytest.mark.parametrize("reduction", ["token", "sequence"])
@pytest.mark.parametrize("kl_coef", [0.0, 0.1])
def test_gradients_that_are_finite_after_the_mean_only(N, reduction, kl_coef):
    """r A and kl_coef exp(ref - logp) past float32 at some tokens, their share of the mean below it. Five
    roundings of the gradient as elsewhere (the powers of two in between are exact)."""
    g = torch.Generator(device=DEV).manual_seed(N)
    old = -torch.rand(N, generator=g, device=DEV)
    logp = old + 0.1 * torch.randn(N, generator=g, device=DEV)
    ref = logp + 0.1 * torch.randn(N, generator=g, device=DEV)
    adv = torch.randn(N, generator=g, device=DEV)
    logp[::7] = old[::7] + 93.0
    adv[::7] = -1.0
    ref[3::7] = logp[3::7] + 95.0
    S = N // 2
    cu = torch.arange(0, N + 1, 2, dtype=torch.int32, device=DEV) if reduction == "sequence" else None
    leaf = logp.detach().requires_grad_(True)
    loss, _, _ = D.policy_loss(leaf, old, adv, ref_logp=ref if kl_coef else None, cu_seqlens=cu, kl_coef=kl_coef,
                               reduction=reduction)
    loss.backward()
    want = P.policy(_np(logp), _np(old), _np(adv), ref=_np(ref) if kl_coef else None,
                    cu=None if cu is None else cu.cpu().numpy(), reduction=reduction, kl_coef=kl_coef)
    assert abs(want[3]).max() * (S if cu is not None else N) > 3.4e38 > abs(want[3]).max()
    got = _np(leaf.grad)
    assert np.all(np.abs(got - want[3]) <= 5 * U * np.abs(want[3]) + 1e-45)


@pytest.mark.parametrize("N", [1, 1000, 9000])
@pytest.mark.parametrize("step", [2.0 ** -22, 2.0 ** -14])
def test_a_policy_next_to_its_reference_keeps_the_digits_of_k(N, step):
    """k = exp(x) - x - 1 for x of a few steps: x^2 / 2 + x^3 / 6 + x^4 / 24 (the rest is below 2^-39 of it)
    to a rounding of the mean and, in 64 bits, an ulp of x in k: 2^-52 / (x / 2) < 2^-29 of k."""
    g = torch.Generator(device=DEV).manual_seed(N)
    logp = -1.0 - torch.randint(0, 2 ** 20, (N,), generator=g, device=DEV).float() * 2.0 ** -21
    ref = logp + torch.randint(1, 8, (N,), generator=g, device=DEV).float() * step
    x = _np(ref) - _np(logp)
    want = (x ** 2 / 2 + x ** 3 / 6 + x ** 4 / 24).mean()
    _, kl, _ = D.policy_loss(logp, logp, torch.zeros_like(logp), ref_logp=ref, kl_coef=0.5)
    assert abs(float(kl) - want) <= (U + 2.0 ** -29) * want
    loss, _, _ = D.policy_loss(logp, logp, torch.zeros_like(logp), ref_logp=ref, kl_coef=0.5)
    assert abs(float(loss) - 0.5 * want) <= (U + 2.0 ** -29) * 0.5 * want


def test_more_sequences_than_a_launch_has_blocks():
    """2^24 and some sequences of 0 to 3 tokens under a mask, their mean of means in 64-bit torch."""
    S = (1 << 24) + 77
    g = torch.Generator(device=DEV).manual_seed(1)
    cu = torch.zeros(S + 1, dtype=torch.int32, device=DEV)
    lens = torch.randint(0, 4, (S,), generator=g, device=DEV)
    cu[1:] = torch.cumsum(lens, 0)
    N = int(cu[-1])
    old = -torch.rand(N, generator=g, device=DEV)
    logp = (old + 0.1 * torch.randn(N, generator=g, device=DEV)).requires_grad_(True)
    adv = torch.randn(N, generator=g, device=DEV)
    mask = torch.rand(N, generator=g, device=DEV) < 0.6
    loss, _, clipped = D.policy_loss(logp, old, adv, mask=mask, cu_seqlens=cu, reduction="sequence")
    got, = torch.autograd.grad(loss, logp)
    owner = torch.repeat_interleave(torch.arange(S, device=DEV), lens)
    count = torch.zeros(S, dtype=torch.float64, device=DEV).index_add_(0, owner, mask.double())
    w = mask.double() / (count[owner].clamp(min=1) * (count > 0).sum())
    r, a = torch.exp(logp.detach().double() - old.double()), adv.double()
    free, bound = r * a, r.clamp(0.8, 1.2) * a
    take = free <= bound
    want = -(w * torch.minimum(free, bound)).sum()
    # 64-bit sums on both sides, terms of size 1
    assert abs(float(loss.detach()) - float(want)) <= U * abs(float(want)) + 1e-9
    assert abs(float(clipped) - float((w * ~take).sum())) <= U + 1e-9
    grad = torch.where(take, -w * free, 0.0)
    assert bool(((got.double() - grad).abs() <= 5 * U * grad.abs() + 1e-45).all())
