"""Verification of rows whose logits are far from 0: the largest takes all, as it does in 64 bits."""

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2608_09703_amd import api as D
from tests.tree_helpers import DEV, tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sampled", [False, True])
@pytest.mark.parametrize("V,top_p,trees", [(300, 0.9, 5), (300, 1.0, 5), (1500, 1.0, 5), (1500, 0.9, 520)])
@pytest.mark.parametrize("scale,base", [(1e7, 0.0), (1e10, 0.0), (1e10, -1e12), (1e20, 0.0), (2e37, 0.0)])
def test_against_the_oracle(scale, base, V, top_p, trees, sampled):
    rng = np.random.default_rng(V + trees)
    n, temperature = 6, 0.7
    parents = tree(rng, trees, n)
    parents[:, 0] = -1
    target = (rng.standard_normal((trees, n, V)) * scale + base).astype(np.float32)
    # the largest is away from the others by more than the rounding of their products with 1 / temperature
    target.reshape(-1, V)[np.arange(trees * n), rng.integers(0, V, trees * n)] = np.float32(5.0 * scale + base)
    draft = target.copy()
    draft[::2] = np.roll(target[::2], 1, axis=2)
    tokens = rng.integers(0, V, (trees, n)).astype(np.int32)
    for b in range(trees):
        for i in range(1, n):
            if 0 <= parents[b, i] < i and rng.random() < 0.7:
                tokens[b, i] = np.argmax(target[b, parents[b, i]])
    ua, us = rng.random((trees, n)).astype(np.float32), rng.random(trees).astype(np.float32)
    gpu = lambda x: torch.tensor(x, device=DEV)  # noqa: E731
    got = D.tree_verify(gpu(target), gpu(tokens), gpu(parents), gpu(ua), gpu(us), draft_logits=gpu(draft) if sampled else None,
                        temperature=temperature, top_p=top_p)
    want = O.verify(target, tokens, parents, ua, us, float(np.float32(temperature)), float(np.float32(top_p)),
                    draft if sampled else None)
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g.cpu().numpy(), w)
    assert want[0].max() > 0
