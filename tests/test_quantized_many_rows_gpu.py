"""More rows than one launch has threads for: 16 threads a row, 2^32 of them a launch."""

import pytest
import torch

from paper_2608_09703_amd import api as D

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


def test_quantize_more_rows_than_a_launch_takes():
    T, d = (1 << 28) + 5, 3
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.randn(T, d, generator=g, device=DEV, dtype=torch.bfloat16)
    q, s = D.quantize_rows(x)
    for at in range(0, T, 1 << 26):  # by the definition, in 64 bits
        y = x[at:at + (1 << 26)].double()
        want_s = (y.abs().amax(1) / 127.0).float()
        assert torch.equal(s[at:at + len(y)], want_s)
        w = want_s.double()[:, None]
        want = torch.where(w > 0, torch.round(y / torch.where(w > 0, w, 1.0)).clamp(-127, 127), 0.0)
        assert torch.equal(q[at:at + len(y)], want.to(torch.int8))
