"""The oracle of tree verification under several children, exactly: at a node the outcome depends on each uniform
through one threshold (acceptance) or a few (the draw), so the distribution of the first token follows from the
thresholds, which bisection finds to the last bits. Whatever tree was drafted, it has to be the verifier's; mistakes
planted in the walk's formula do not keep it."""

import inspect
import itertools

import numpy as np
import pytest

from oracle import decode as C
from oracle import tree as O

MUTANTS = {
    "residual_not_kept": ("p = left / left.sum()", "pass"),
    "residual_not_normalised": ("p = left / left.sum()", "p = left"),
    "half_of_q": ("np.maximum(p - q, 0.0)", "np.maximum(p - 0.5 * q, 0.0)"),
    "turned_down_token_stays": ("left[x] = 0.0", "pass"),
    "accepts_without_q": ("float(u_accept[b][i]) * qx < px", "float(u_accept[b][i]) < px"),
}


def _mutant(name):
    old, new = MUTANTS[name]
    src = inspect.getsource(O.verify)
    assert src.count(old) == 1
    scope = dict(vars(O))
    exec(src.replace(old, new), scope)
    return scope["verify"]


def _border(f):
    """The u in [0, 1] up to which f is true (f is true below it alone)."""
    if not f(0.0):
        return 0.0
    lo, hi = 0.0, 1.0  # (1 itself is no uniform)
    for _ in range(60):
        mid = 0.5 * (lo + hi)
        lo, hi = (mid, hi) if f(mid) else (lo, mid)
    return hi


def _first_token(verify, target, draft, children):
    """The distribution of the token after node 0 over all uniforms, for one drafted list of children."""
    V, n = target.shape[-1], len(children) + 1
    parents = np.array([[-1] + [0] * (n - 1)])
    tokens = np.array([[0] + list(children)])
    run = lambda ua, us: verify(target, tokens, parents, np.array([ua]), np.array([us]), 1.0, 1.0, draft)  # noqa: E731
    out, left = np.zeros(V), 1.0
    for j in range(1, n):
        t = _border(lambda u: run([2.0] * j + [u] + [2.0] * (n - 1 - j), 0.5)[1][0, 1] == j)
        out[children[j - 1]] += left * t
        left *= 1.0 - t
    if left > 0:
        edges = [0.0] + [_border(lambda u: run([2.0] * n, u)[2][0] <= v) for v in range(V)]
        out += left * np.diff(edges)
    return out


def _sampled(verify):
    """Three children, each drawn from q: the mean over all that can be drawn. Of p - q one
    token's is above q and another's between 0 and q: only there does the mass of what is left matter."""
    V = 4
    target = np.log(np.array([0.6, 0.3, 0.05, 0.05]))[None, None].repeat(4, 1)
    draft = np.log(np.array([0.2, 0.2, 0.3, 0.3]))[None, None].repeat(4, 1)
    q = C.filtered_probs(draft[0, 0], 1.0, 1.0)
    got = sum(np.prod(q[list(c)]) * _first_token(verify, target, draft, c) for c in itertools.product(range(V), repeat=3))
    return got, C.filtered_probs(target[0, 0], 1.0, 1.0)


def _proposed(verify):
    """Four children without probabilities, one of them twice."""
    V = 6
    target = (np.random.default_rng(4).standard_normal((1, 5, V)) * 1.5).astype(np.float32)
    return _first_token(verify, target, None, (4, 1, 4, 0)), C.filtered_probs(target[0, 0], 1.0, 1.0)


# 60 halvings leave 2^-60 of a border, sums and products of some dozen numbers near 1 a few 2^-52 each
TOL = 1e-12


@pytest.mark.parametrize("dist", [_sampled, _proposed])
def test_first_token_is_the_verifiers(dist):
    got, want = dist(O.verify)
    np.testing.assert_allclose(got, want, atol=TOL)


@pytest.mark.parametrize("name,dist", [
    ("residual_not_kept", _sampled), ("residual_not_normalised", _sampled), ("half_of_q", _sampled),
    ("accepts_without_q", _sampled), ("residual_not_kept", _proposed), ("residual_not_normalised", _proposed),
    ("turned_down_token_stays", _proposed)])
def test_planted_mistakes_are_seen(name, dist):
    got, want = dist(_mutant(name))
    assert np.abs(got - want).max() > 1e-3


def test_thresholds_without_probabilities():
    """Child j of p_1, p_2, .. is taken below p_j / (1 - p_1 - .. - p_(j-1))."""
    p = np.array([0.4, 0.2, 0.12, 0.08, 0.15, 0.05])
    target = np.log(p)[None, None].repeat(5, 1)
    for j in range(1, 5):
        t = _border(lambda u: O.verify(target, np.array([[0, 0, 1, 2, 3]]), np.array([[-1, 0, 0, 0, 0]]),
                                       np.array([[2.0] * j + [u] + [2.0] * (4 - j)]), np.array([0.5]), 1.0, 1.0)[1][0, 1] == j)
        assert abs(t - p[j - 1] / (1.0 - p[:j - 1].sum())) < TOL
