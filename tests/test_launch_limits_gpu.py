"""More rows and tokens than one launch has threads for."""

import pytest
import torch

from paper_2608_09703_amd import api as D

DEV = "cuda:0"
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("greedy", [True, False])
def test_sampled_rows(greedy):
    rows, V = (1 << 22) + 7, 4  # 1,024 threads a row
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    logits = torch.randn(rows, V, generator=g, device=DEV)
    u = torch.rand(rows, generator=g, device=DEV)
    tok = D.sample(logits, None if greedy else u, greedy=greedy)
    if greedy:
        assert torch.equal(tok, logits.argmax(1).to(torch.int32))
        return
    c = logits.double().softmax(1).cumsum(1)
    want = (c <= u.double()[:, None]).sum(1).clamp(max=V - 1).to(torch.int32)
    # a uniform within float32's roundings of a border may fall to either side: some 2^-22 of each of 3 borders
    off = tok != want
    near = (c - u.double()[:, None]).abs().amin(1) < 2.0 ** -21
    assert not (off & ~near).any() and off.sum() < 100


def test_label_logits():
    T, V, d = (1 << 25) + 9, 16, (8, 8)  # 64 threads for each of two sub-models' tokens
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    h = [torch.randn(T, k, generator=g, device=DEV, dtype=torch.bfloat16) for k in d]
    W = [torch.randn(V, k, generator=g, device=DEV, dtype=torch.bfloat16) for k in d]
    y = torch.randint(0, V, (T,), generator=g, device=DEV)
    with torch.no_grad():
        ce, _, _ = D.distill(h, W, y)
    for i in range(2):
        want = torch.zeros((), dtype=torch.float64, device=DEV)
        for at in range(0, T, 1 << 22):
            z = h[i][at:at + (1 << 22)].double() @ W[i].double().t()
            want += torch.nn.functional.cross_entropy(z, y[at:at + (1 << 22)], reduction="sum")
        # each token's loss in float32, a few 2^-24 of numbers below 32
        torch.testing.assert_close(ce[i].double(), want / T, rtol=1e-5, atol=0.0)
