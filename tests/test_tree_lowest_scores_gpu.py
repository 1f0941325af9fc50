"""Scores next to float32's lowest number, which a row's maximum starts from."""

import numpy as np
import pytest
import torch

from paper_2608_09703_amd import api as D

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def test_scores_at_the_lowest_number():
    """Scores whose product with the scale is float32's lowest number itself: they weigh alike."""
    Dh = 32
    low = np.float32(np.finfo(np.float32).min)
    scale = np.float32(0.9)
    by = float(np.float32(scale * np.float32(1.4426950408889634)))
    z = np.float32(float(low) / by)
    near = [z]
    for away in (-np.inf, np.inf):  # the neighbours whose rounded product is the lowest number too
        x = z
        for _ in range(3):
            x = np.nextafter(x, np.float32(away))
            near.append(x)
    with np.errstate(over="ignore"):
        keys = [x for x in near if np.float32(float(x) * by) == low]
    assert keys
    for x in keys:
        k = torch.zeros(2, 1, 16, Dh, device=DEV)
        k[0, 0, :, 0] = float(x)
        v = torch.zeros_like(k)
        v[0, 0, :, 1] = torch.arange(16.0, device=DEV)
        q = torch.zeros(1, 1, 1, Dh, device=DEV)
        q[..., 0] = 1.0
        table = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
        lengths = torch.tensor([15], dtype=torch.int32, device=DEV)
        got = D.tree_attention(q, k, v, table, lengths, scale=float(scale))
        assert got[0, 0, 0, 1].item() == 7.5, x
