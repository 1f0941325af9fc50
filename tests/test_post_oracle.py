"""Pins of the float64 oracle of the post-training operators: central differences of
its own forward, and PyTorch's float64 autograd of the plain formulas."""

import numpy as np
import pytest
import torch

from oracle import post as P


def _differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_layer_norm_gradients_are_its_differences():
    r = np.random.default_rng(0)
    x, w, b, gy = r.normal(size=(3, 7)) + 2.0, r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    gx, gw, gb = P.layer_norm_backward(x, w, gy, eps=0.1)
    np.testing.assert_allclose(gx, _differences(lambda v: (P.layer_norm(v, w, b, 0.1) * gy).sum(), x), atol=1e-8)
    np.testing.assert_allclose(gw, _differences(lambda v: (P.layer_norm(x, v, b, 0.1) * gy).sum(), w), atol=1e-8)
    np.testing.assert_allclose(gb, _differences(lambda v: (P.layer_norm(x, w, v, 0.1) * gy).sum(), b), atol=1e-8)


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_token_logp_gradients_are_its_differences(temperature):
    r = np.random.default_rng(1)
    h, W, g = r.normal(size=(5, 4)), r.normal(size=(6, 4)), r.normal(size=5)
    tokens = np.array([2, -100, 0, 9, 5])  # one ignored, one out of range
    gh, gW = P.token_logp_backward(h, W, tokens, g, temperature)
    f = lambda a, b: (P.token_logp(a, b, tokens, temperature)[0] * g).sum()  # noqa: E731
    np.testing.assert_allclose(gh, _differences(lambda v: f(v, W), h), atol=1e-8)
    np.testing.assert_allclose(gW, _differences(lambda v: f(h, v), W), atol=1e-8)
    logp, entropy = P.token_logp(h, W, tokens, temperature)
    d = torch.distributions.Categorical(logits=torch.tensor(h @ W.T / temperature))
    ok = [0, 2, 4]
    np.testing.assert_allclose(logp[ok], d.log_prob(torch.tensor([2, 0, 0, 0, 5])).numpy()[ok], rtol=1e-12)
    np.testing.assert_allclose(entropy[ok], d.entropy().numpy()[ok], rtol=1e-12)
    assert not logp[[1, 3]].any() and not entropy[[1, 3]].any() and not gh[[1, 3]].any()


@pytest.mark.parametrize("reduction", ["token", "sequence"])
@pytest.mark.parametrize("per_sequence", [False, True])
def test_policy_gradient_is_its_differences(reduction, per_sequence):
    r = np.random.default_rng(2)
    n, cu = 12, [1, 4, 4, 11]
    logp, old, ref = (r.normal(size=n) * 0.3 for _ in range(3))
    adv = r.normal(size=3 if per_sequence else n)
    mask = r.random(n) < 0.7
    args = dict(ref=ref, mask=mask, cu=cu, per_sequence=per_sequence, kl_coef=0.3, reduction=reduction)
    grad = P.policy(logp, old, adv, **args)[3]
    np.testing.assert_allclose(grad, _differences(lambda v: P.policy(v, old, adv, **args)[0], logp), atol=1e-8)
    assert grad[0] == 0 and grad[11] == 0 and not grad[~mask].any()


def test_policy_without_a_counted_token_and_clip():
    z = np.zeros(3)
    assert P.policy(z, z, z, mask=[False] * 3)[:3] == (0.0, 0.0, 0.0)
    norm, out = P.clip([np.array([3.0]), np.array([[4.0]])], 1.0)
    assert norm == 5.0 and out[0][0] == pytest.approx(0.6) and out[1][0, 0] == pytest.approx(0.8)
    assert P.clip([np.array([3.0])], 4.0)[1][0][0] == 3.0
