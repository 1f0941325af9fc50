"""The post-training operators together, as a step uses them: a norm in front of the
head, log-probabilities under the policy and the frozen reference, the policy loss,
its backward through all of them, and the clipping of the gradients.
"""

import numpy as np
import pytest
import torch

from oracle import post as P
from paper_2608_09703_amd import api as D
from tests.grad_checks import assert_grad_rows

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _np(x):
    return x.detach().double().cpu().numpy()


class _Step:
    def __init__(self, dtype, seed=0, T=220, d=96, V=700):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.x = (r(T, d) + 0.2).to(dtype)
        self.w = 1 + 0.1 * r(d)
        self.b = 0.1 * r(d)
        self.W = (r(V, d) * 0.2).to(dtype)
        self.W_ref = (self.W.float() + 0.02 * r(V, d)).to(dtype)
        self.tokens = torch.randint(0, V, (T,), generator=g, device=DEV)
        self.tokens[::7] = -100
        self.cu = torch.tensor([0, 60, 61, 200], dtype=torch.int32, device=DEV)
        self.adv = r(3)
        self.mask = self.tokens != -100
        self.temperature, self.kl_coef, self.max_norm = 0.9, 0.05, 0.01
        with torch.no_grad():
            h = D.layer_norm(self.x, self.w, self.b)
            self.ref = D.token_logp(h, self.W_ref, self.tokens, temperature=self.temperature)[0]
            self.old = D.token_logp(h, self.W, self.tokens, temperature=self.temperature)[0] + 0.1 * r(T)
        self.leaves = [t.requires_grad_(True) for t in (self.x, self.w, self.b, self.W)]

    def run(self):
        h = D.layer_norm(self.x, self.w, self.b)
        logp, entropy = D.token_logp(h, self.W, self.tokens, temperature=self.temperature)
        loss, kl, clipped = D.policy_loss(logp, self.old, self.adv, ref_logp=self.ref, mask=self.mask,
                                          cu_seqlens=self.cu, per_sequence=True, clip_low=0.1, clip_high=0.1,
                                          kl_coef=self.kl_coef, reduction="sequence")
        grads = list(torch.autograd.grad(loss, self.leaves))
        norm = D.clip_grad_norm(grads, self.max_norm)
        return [loss.detach(), kl, clipped, norm, logp.detach(), entropy] + grads


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_step_against_64_bits(dtype):
    s = _Step(dtype)
    loss, kl, clipped, norm, logp, entropy, *grads = s.run()
    x, w, b, W = (_np(t) for t in s.leaves)
    h = P.layer_norm(x, w, b)
    tokens = s.tokens.cpu().numpy()
    lp, _ = P.token_logp(h, W, tokens, s.temperature)
    # bf16: the normalised rows are rounded before the head, half a step of 2^-8 of each of 96
    # entries, times a head row of length 0.2 sqrt(96) / temperature: 2^-8 * 0.2 * 96 / 0.9 < 0.09 at the
    # very most, and twice that with the log-sum-exp
    np.testing.assert_allclose(_np(logp), lp, atol=5e-5 if dtype == torch.float32 else 0.17)
    # from here on the loss's own inputs
    want = P.policy(_np(logp), _np(s.old), _np(s.adv), ref=_np(s.ref), mask=s.mask.cpu().numpy(),
                    cu=s.cu.cpu().numpy(), per_sequence=True, clip_low=0.1, clip_high=0.1, kl_coef=s.kl_coef,
                    reduction="sequence")
    for got, ref in zip((loss, kl, clipped), want):
        assert abs(float(got) - ref) <= 1e-6 * abs(ref) + 1e-9
    hr = _np(D.layer_norm(s.x.detach(), s.w.detach(), s.b.detach()))  # as the head read it
    gh, gW = P.token_logp_backward(hr, W, tokens, want[3], s.temperature)
    gx, gw, gb = P.layer_norm_backward(x, w, gh)
    ref_norm, ref = P.clip([gx, gw, gb, gW], s.max_norm)
    # the parameters' sums over tokens cancel, so their roundings count against the largest of them
    tol = 1e-4 if dtype == torch.float32 else 2e-2
    assert ref_norm > s.max_norm and abs(float(norm) - ref_norm) <= tol * ref_norm
    for g, r, name in zip(grads, ref, ("x", "w", "b", "W")):
        if r.ndim == 2:
            assert_grad_rows(_np(g), r, name, rtol=2e-2)
        else:
            assert np.abs(_np(g) - r).max() <= 4 * tol * np.abs(r).max(), name
    total = np.sqrt(sum((_np(g) ** 2).sum() for g in grads))
    assert abs(total - s.max_norm) <= 1e-3 * s.max_norm


def test_gradients_of_gradients_are_refused():
    x = torch.randn(4, 64, device=DEV, requires_grad=True)
    W = torch.randn(9, 64, device=DEV, requires_grad=True)
    logp = torch.randn(4, device=DEV, requires_grad=True)
    y = D.layer_norm(x, torch.ones(64, device=DEV))
    lp, _ = D.token_logp(x, W, torch.zeros(4, dtype=torch.int64, device=DEV))
    loss, _, _ = D.policy_loss(logp, torch.zeros(4, device=DEV), torch.ones(4, device=DEV))
    for out, leaf in ((y.sum(), x), (lp.sum(), W), (loss, logp)):
        with pytest.raises(RuntimeError, match="gradients of gradients"):
            torch.autograd.grad(out, leaf, create_graph=True)


def test_step_on_another_stream_has_the_same_bits():
    s = _Step(torch.bfloat16)
    ref = s.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(ref, got):
        assert torch.equal(a, b)


def test_step_with_saved_tensors_on_the_host_has_the_same_bits():
    s = _Step(torch.bfloat16)
    ref = s.run()
    with torch.autograd.graph.save_on_cpu():
        got = s.run()
    for a, b in zip(ref, got):
        assert torch.equal(a, b)


def test_two_steps_at_once():
    """On two streams, each with its own tensors but the same head."""
    steps = [_Step(torch.bfloat16, seed=k) for k in (1, 2)]
    steps[1].W = steps[1].leaves[3] = steps[0].W
    ref = [s.run() for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = []
    for s, q in zip(steps, streams):
        with torch.cuda.stream(q):
            got.append(s.run())
    torch.cuda.synchronize()
    for a, b in zip(ref, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_step_replays(dtype):
    """Two graphs of the step replayed in turn, with eager work in between, after new inputs."""
    print(f"[post-training step] capture, {dtype}", flush=True)
    s = _Step(dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = s.run()
        graphs.append((g, out))
    for rep in range(4):
        print(f"[post-training step] replay {rep}", flush=True)
        with torch.no_grad():
            s.x.mul_(1.01)
            s.adv.neg_()
            # other tokens, and another number of them that count
            s.tokens.copy_(torch.roll(s.tokens, 5))
            s.tokens[rep * 11:rep * 30] = -100
            s.mask.copy_(s.tokens != -100)
        ref = s.run()
        for g, out in graphs if rep % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for k, (a, b) in enumerate(zip(ref, out)):
                assert torch.equal(a, b), (rep, k)
