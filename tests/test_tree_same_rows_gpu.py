"""Verification where the draft's rows are the verifier's: nothing is left of p - q, and what is drawn after children that
neither could produce comes from p."""

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2608_09703_amd import api as D
from paper_2608_09703_amd import binding as B

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("records", [False, True])
@pytest.mark.parametrize("shift", [0.0, 8.0])
@pytest.mark.parametrize("V,top_p,trees", [(2, 1.0, 7), (60, 0.9, 7), (700, 0.97, 7), (700, 1.0, 7), (3000, 1.0, 7), (3000, 0.999, 7),
                                           (700, 0.97, 520), (3000, 1.0, 520)])
def test_children_out_of_range(V, top_p, trees, shift, records):
    rng = np.random.default_rng(V + trees)
    n, temperature = 5, 0.5
    # multiples of 2^-10, so that a shift by 8 changes no difference
    target = (np.round(rng.standard_normal((trees, n, V)) * 2048) / 1024).astype(np.float32)
    draft = target + np.float32(shift)
    parents = np.tile(np.array([-1, 0, 0, 1, 0], np.int32), (trees, 1))
    tokens = np.tile(np.array([0, -1, V, 0, 2 ** 31 - 1], np.int32), (trees, 1))
    if trees % 2 == 1:  # the last child can be produced, after two that cannot
        tokens[::2, 4] = target[::2, 0].argmax(1)
    ua, us = rng.random((trees, n)).astype(np.float32), rng.random(trees).astype(np.float32)
    gpu = lambda x: torch.tensor(x, device=DEV)  # noqa: E731
    kw = dict(temperature=temperature, top_p=top_p)
    rec = None
    if records:
        rec = torch.empty(trees * n * B.ROW_PARAMS_BYTES, dtype=torch.uint8, device=DEV)
        D.sample(gpu(draft).view(trees * n, V), torch.zeros(trees * n, device=DEV), params=rec, **kw)
    got = D.tree_verify(gpu(target), gpu(tokens), gpu(parents), gpu(ua), gpu(us), draft_logits=gpu(draft), draft_params=rec, **kw)
    want = O.verify(target, tokens, parents, ua, us, temperature, float(np.float32(top_p)), target)
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g.cpu().numpy(), w)
