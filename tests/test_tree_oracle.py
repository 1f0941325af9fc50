"""Pins of oracle/tree.py: against the chain's definition, the sampled distribution, and a direct softmax."""

import numpy as np
import pytest

from oracle import decode as C
from oracle import tree as O


def _rows(rng, *shape):
    return (rng.standard_normal(shape) * 2).astype(np.float32)


def test_attention_is_a_softmax_over_what_a_node_sees():
    rng = np.random.default_rng(10)
    B, n, heads, D, L = 1, 6, 4, 8, 5
    parents = np.array([[-1, 0, 0, 1, -2, 4]])
    q, k, v = rng.standard_normal((B, n, heads, D)), rng.standard_normal((B, L + n, 2, D)), rng.standard_normal((B, L + n, 2, D))
    got = O.attention(q, k, v, [L], parents)
    for i, sees in enumerate([[0], [0, 1], [0, 2], [0, 1, 3], None, None]):
        for h in range(heads):
            if sees is None:
                assert (got[0, i, h] == 0).all()
                continue
            at = list(range(L)) + [L + j for j in sees]
            s = k[0, at, h // 2] @ q[0, i, h] / np.sqrt(D)
            w = np.exp(s - s.max())
            np.testing.assert_allclose(got[0, i, h], (w / w.sum()) @ v[0, at, h // 2], rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("sampled", [True, False])
def test_tokens_follow_the_verifiers_distribution(sampled):
    """The first token after node 0, exactly: the uniforms of a tree of three children on a fine grid."""
    rng = np.random.default_rng(5)
    V, m = 5, 24
    target, draft = _rows(rng, 1, 4, V), _rows(rng, 1, 4, V)
    p, q = C.filtered_probs(target[0, 0], 1.0, 1.0), C.filtered_probs(draft[0, 0], 1.0, 1.0)
    parents = np.array([[-1, 0, 0, 0]])
    grid = (np.arange(m) + 0.5) / m
    total = np.zeros(V)
    # two children, both acceptance uniforms and the draw's in one grid each
    parents, target, draft = parents[:, :3], target[:, :3], draft[:, :3]
    pairs = [(a, b) for a in range(V) for b in range(V)] if sampled else [(1, 3)]
    for a, b in pairs:
        weight = q[a] * q[b] if sampled else 1.0
        tokens = np.array([[0, a, b]])
        for u1 in grid:
            for u2 in grid:
                ua = np.array([[0, u1, u2]], np.float32)
                hist = np.zeros(V)
                first = O.verify(target, tokens, parents, ua, np.array([0.5], np.float32), 1.0, 1.0, draft if sampled else None)
                if first[0][0] > 0:
                    hist[tokens[0, first[1][0][1]]] = 1.0
                else:
                    for us in grid:
                        r = O.verify(target, tokens, parents, ua, np.array([us], np.float32), 1.0, 1.0, draft if sampled else None)
                        hist[r[2][0]] += 1.0 / m
                total += weight * hist / m ** 2
    # each of the three grids misplaces at most one cell at each of its borders: 1 / m an acceptance, V / m the draw
    assert abs(total.sum() - 1) < 1e-9
    np.testing.assert_allclose(total, p, atol=3.0 / m)


def test_rows_as_integers():
    x = np.array([[127.0, -3.5, 2.5, 0.49], [0, 0, 0, 0]])
    q, s = O.quantize(x)
    assert s.tolist() == [1.0, 0.0] and q.tolist() == [[127, -4, 2, 0], [0, 0, 0, 0]]
