"""Token log-probabilities of a head on the GPU against the float64 oracle.

Forward: fp32 rows, the statistics' tolerance of the fused loss (5e-5 for a
log-sum-exp and a logit of fp32 sums). Gradients: every row within the fused loss's
gradient bounds (the logit gradient is bf16 in between on the bf16 path), and
element by element within what the roundings allow: with G the exact logit gradient,
2^-8 sum |G| |W| for its rounding (of its entries over the own token's one), for grad_W
2^-8 sum |G| |h| more for the rounding of the scaled hidden states (and the product of
both, 2^-16), 2^-8 of the result for the output's, and
2^-12 sum |G| |W| for the recomputed logits (a logit of fp32 sums is off by less than
2^-13 here, and exp turns that into a relative error of G's softmax part). A kept
logit's distance below a maximum, over tau, is off by half a step of 32 / 65535, and so
the softmax entry p by 2^-12 p (1.01 of it, with exp's second order); entries further than
32 below count as e^-32 of the maximum's. E in the check is what that adds to G.
"""

import numpy as np
import pytest
import torch

from oracle import post as P
from paper_2608_09703_amd import api as D
from paper_2608_09703_amd import binding as B
from tests.grad_checks import assert_grad_rows

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _np(x):
    return x.detach().double().cpu().numpy()


def _draw(T, d, V, dtype, seed, ignore=0.2):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(T, d, generator=g, device=DEV).to(dtype)
    W = (torch.randn(V, d, generator=g, device=DEV) * (2.0 / d ** 0.5)).to(dtype)
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV)
    tokens[torch.rand(T, generator=g, device=DEV) < ignore] = -100
    gl = torch.randn(T, generator=g, device=DEV)
    return h, W, tokens, gl


def _check(h, W, tokens, gl, temperature, got, what):
    logp, entropy, gh, gW = got
    hn, Wn, tn, gn = _np(h), _np(W), tokens.cpu().numpy(), _np(gl)
    lp, en = P.token_logp(hn, Wn, tn, temperature)
    np.testing.assert_allclose(_np(logp), lp, rtol=1e-5, atol=5e-5, err_msg=what)
    np.testing.assert_allclose(_np(entropy), en, rtol=1e-5, atol=5e-5, err_msg=what)
    rh, rW = P.token_logp_backward(hn, Wn, tn, gn, temperature)
    bf16 = h.dtype == torch.bfloat16
    rows = np.flatnonzero((tn != -100) & (tn >= 0) & (tn < len(Wn)))
    G = np.zeros((len(hn), len(Wn)))
    if rows.size:
        z = hn[rows] @ Wn.T / temperature
        p = np.exp(z - z.max(1, keepdims=True))
        G[rows] = p / p.sum(1, keepdims=True)
        G[rows, tn[rows]] = 1 - G[rows, tn[rows]]
        G[rows] *= np.abs(gn[rows])[:, None] / temperature
    rel = 2.0 ** -8 + 2.0 ** -12 if bf16 else 2.0 ** -12
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    E = np.zeros_like(G)
    if bf16 and rows.size:
        E[rows] = (1.01 * 2.0 ** -12 * p / p.sum(1, keepdims=True) + np.exp(-32.0)) * np.abs(gn[rows])[:, None] / temperature
    rel_W = rel + 2.0 ** -8 + 2.0 ** -16 if bf16 else rel
    for g, r, s, e, name in ((gh, rh, rel * (G @ np.abs(Wn)), E @ np.abs(Wn), "grad_h"),
                             (gW, rW, rel_W * (G.T @ np.abs(hn)), E.T @ np.abs(hn), "grad_W")):
        if g is None:
            continue
        gn_ = _np(g)
        bad = ~(np.abs(gn_ - r) <= s + e + half * np.abs(r))
        assert not bad.any(), f"{what} {name}: {bad.sum()} off, first at {np.argwhere(bad)[0]}"
        assert_grad_rows(gn_, r, f"{what} {name}")
    return rh, rW


def _run(h, W, tokens, gl, **kw):
    h, W = h.detach().requires_grad_(True), W.detach().requires_grad_(True)
    logp, entropy = D.token_logp(h, W, tokens, **kw)
    gh, gW = torch.autograd.grad(logp, (h, W), gl)
    return logp, entropy, gh, gW


SHAPES = [(1, 8, 2), (1, 64, 300), (2, 64, 128), (127, 64, 129), (128, 72, 1000), (129, 200, 515), (300, 128, 2000),
          (257, 520, 4097), (700, 1024, 3001), (129, 2048, 255), (300, 2080, 1029)]


@pytest.mark.parametrize("T,d,V", SHAPES)
@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("dtype,keep", [(torch.bfloat16, True), (torch.bfloat16, False), (torch.float32, False)])
def test_shapes(T, d, V, temperature, dtype, keep):
    h, W, tokens, gl = _draw(T, d, V, dtype, T + d)
    got = _run(h, W, tokens, gl, temperature=temperature, keep_logits=keep)
    _check(h, W, tokens, gl, temperature, got, f"{T} {d} {V}")


@pytest.mark.parametrize("d", [64, 200, 2048])
def test_kept_logits(d, monkeypatch):
    """Kept by themselves up to a size; read, not written, by the backward."""
    h, W, tokens, gl = _draw(300, d, 1500, torch.bfloat16, d)
    h, W = h.requires_grad_(True), W.requires_grad_(True)

    def grads(times=1, **kw):
        logp, _ = D.token_logp(h, W, tokens, **kw)
        return [logp.detach()] + [torch.autograd.grad(logp, (h, W), gl, retain_graph=True) for _ in range(times)]
    kept, first, second = grads(2, keep_logits=True)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    assert all(torch.equal(a, b) for a, b in zip(first, grads()[1]))
    again = grads(keep_logits=False)
    assert torch.equal(kept, again[0]) and not torch.equal(first[1], again[1][1])
    monkeypatch.setattr(D, "KEEP_LOGITS_BYTES", 1000)
    assert all(torch.equal(a, b) for a, b in zip(again[1], grads()[1]))


@pytest.mark.parametrize("d,rec", [(64, 64), (2048, 128)])
def test_what_is_kept_of_a_logit(d, rec):
    """Rows of 16 bits: the nearest 65,535th of 32 to the distance below the record's maximum, over tau."""
    T, V, tau = 300, 700, 0.5
    h = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV)
    h[:, 0] = torch.linspace(0.25, 1.5, T)
    W = torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    W[:, 0] = torch.randn(V, device=DEV) * 4
    W[::90, 0] = -40.0
    tokens = torch.zeros(T, dtype=torch.int64, device=DEV)
    p = D.make_problem([h], [W], tokens, tau=tau)
    fwd, _, size = B.token_logp_workspace(p)
    kept = torch.zeros(size, dtype=torch.uint8, device=DEV)
    ws = torch.empty(fwd, dtype=torch.uint8, device=DEV)
    stats = torch.empty(B.query_sizes(p)[1], dtype=torch.uint8, device=DEV)
    logp = torch.empty(T, device=DEV)
    B.token_logp_fwd(p, stats.data_ptr(), logp.data_ptr(), None, kept.data_ptr(), ws.data_ptr(), fwd,
                     D._stream(h.device))
    ld = (V + 255) // 256 * 256
    got = kept[:2 * T * ld].cpu().numpy().view(np.uint16).reshape(T, ld)[:, :V].astype(np.float64)
    z = _np(h)[:, :1] * _np(W)[:, 0]  # exact: products of two bf16 numbers
    for v0 in range(0, V, rec):
        x = (z[:, v0:v0 + rec].max(1, keepdims=True) - z[:, v0:v0 + rec]) / tau / 32 * 65535
        # half a step, and three fp32 roundings of a value up to 65535
        assert np.abs(got[:, v0:v0 + rec] - np.minimum(x, 65535)).max() <= 0.5 + 3 * 65535 * 2.0 ** -24


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_few_tokens_keep_their_digits(T, keep):
    """The token's own entry of the logit gradient carries grad_h and the own rows of grad_W: it is not
    rounded, so what is left is one rounding of each element (relative rms 2^-8 / sqrt(3) at most, where
    roundings were uniform) and 2^-12 of the softmax; a rounded entry would add up to 2^-8 to all at once."""
    h, W, tokens, gl = _draw(T, 512, 4000, torch.bfloat16, 20 + T, ignore=0.0)
    logp, _, gh, gW = _run(h, W, tokens, gl, keep_logits=keep)
    rh, rW = P.token_logp_backward(_np(h), _np(W), tokens.cpu().numpy(), _np(gl))
    for g, r, name in ((gh, rh, "grad_h"), (gW, rW, "grad_W")):
        rows = np.unique(tokens.cpu().numpy()) if name == "grad_W" else slice(None)
        e = np.linalg.norm(_np(g)[rows] - r[rows], axis=1) / np.linalg.norm(r[rows], axis=1)
        assert e.max() <= 2.0 ** -8 / 3 ** 0.5 + 2.0 ** -11, (name, e)


def test_a_token_that_is_nearly_certain():
    """1 - p from the log-probability: gradients of confident tokens keep their size."""
    h, W, tokens, gl = _draw(64, 256, 1000, torch.bfloat16, 30, ignore=0.0)
    W[tokens] += (h.float() * 0.05).to(W.dtype)
    logp, _, gh, gW = _run(h, W, tokens, gl)
    lp = P.token_logp(_np(h), _np(W), tokens.cpu().numpy())[0]
    assert np.median(lp) > -0.1
    rh, rW = P.token_logp_backward(_np(h), _np(W), tokens.cpu().numpy(), _np(gl))
    # one rounding of each element, one of each softmax entry over 1 - p (2^-8 at most, of entries that add up
    # to 1 like the own token's), and 1 - p is off by logp's error, under 2^-18 for logits of 16: 2^-10 of 2^-8
    z = 1 - np.exp(lp)
    n = np.linalg.norm
    ok = z > 2.0 ** -8
    e = n(_np(gh) - rh, axis=1) / n(rh, axis=1)
    assert ok.any() and e[ok].max() <= 2.0 ** -8 + 2.0 ** -10


def test_kept_logits_are_freed_by_the_backward():
    T, d, V = 2000, 64, 20000
    h, W, tokens, gl = _draw(T, d, V, torch.bfloat16, 13)
    W.requires_grad_(True)
    used = torch.cuda.memory_allocated
    before = used()
    logp, entropy = D.token_logp(h, W, tokens)
    assert used() - before >= 2 * T * V
    gW = torch.autograd.grad(logp, W, gl)
    assert used() - before < T * V and logp.requires_grad
    del gW
    with torch.no_grad():
        before = used()
        logp = D.token_logp(h, W, tokens)
        assert used() - before < T * V


@pytest.mark.parametrize("T,d,V,chunk", [(20001, 64, 130, 0), (3000, 64, 3001, 256), (1000, 2048, 5003, 1280)])
def test_kept_logits_over_many_tokens_and_chunks(T, d, V, chunk):
    h, W, tokens, gl = _draw(T, d, V, torch.bfloat16, 14, ignore=0.4)
    got = _run(h, W, tokens, gl, temperature=1.3, vocab_chunk=chunk, keep_logits=True)
    _check(h, W, tokens, gl, 1.3, got, f"{T} {d} {V}")


@pytest.mark.parametrize("keep", [True, False])
def test_far_logits(keep):
    """Logits hundreds apart: entries that the softmax leaves nothing of, and distances past what is kept."""
    h, W, tokens, gl = _draw(130, 64, 1000, torch.bfloat16, 15)
    h[::3] *= 30
    h[1::3] *= 3e4
    logp, entropy, gh, gW = _run(h, W, tokens, gl, keep_logits=keep)
    rh, rW = P.token_logp_backward(_np(h), _np(W), tokens.cpu().numpy(), _np(gl))
    # (a logit of size 1e5 is off by 1e-2 itself: rows near a tie are left to the others)
    assert torch.isfinite(logp).all() and torch.isfinite(gh).all() and torch.isfinite(gW).all()
    assert_grad_rows(_np(gh)[::3], rh[::3], "grad_h")
    assert_grad_rows(_np(gh)[2::3], rh[2::3], "grad_h")


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 96), (torch.bfloat16, 2048), (torch.float32, 96)])
@pytest.mark.parametrize("kept", [[], [0], [299], [5, 130, 299], list(range(0, 300, 2)), list(range(200, 300))],
                         ids=lambda v: f"{len(v)}kept")
def test_ignored_tokens(kept, dtype, d):
    """From every token ignored to half of them in turn; the others' values do not matter."""
    h, W, tokens, gl = _draw(300, d, 700, dtype, 3, ignore=0.0)
    ignored = torch.ones(300, dtype=torch.bool, device=DEV)
    ignored[kept] = False
    tokens[ignored] = -100
    got = _run(h, W, tokens, gl)
    _check(h, W, tokens, gl, 1.0, got, f"{len(kept)} kept")
    for g in (got[0], got[1], got[2]):
        assert not g[ignored].any()
    h[ignored] = float("nan")
    h[ignored.nonzero()[::2, 0]] = float("-inf")
    gl[ignored] = float("inf")
    for a, b in zip(got, _run(h, W, tokens, gl)):
        assert torch.equal(a, b)


def test_tokens_out_of_range_are_ignored_and_flagged():
    h, W, tokens, gl = _draw(200, 64, 500, torch.bfloat16, 4)
    tokens[3], tokens[7] = 500, -1
    got = _run(h, W, tokens, gl)
    _check(h, W, tokens, gl, 1.0, got, "out of range")
    p = D.make_problem([h], [W], tokens)
    buf = D.Buffers(p, h.device)
    ws = torch.empty(B.token_logp_workspace(p)[0], dtype=torch.uint8, device=DEV)
    logp = torch.empty(200, device=DEV)

    def flags():
        B.token_logp_fwd(p, buf.stats.data_ptr(), logp.data_ptr(), None, None, ws.data_ptr(), ws.numel(),
                         D._stream(h.device))
        n, f = B.read_stats_header(p, buf.stats.data_ptr(), D._stream(h.device))
        assert n == int(((tokens >= 0) & (tokens < 500)).sum()) and f == B.device_error(
            p, buf.stats.data_ptr(), D._stream(h.device))
        return f
    assert flags() == B.MLS_DEVFLAG_LABEL_RANGE
    tokens[3] = tokens[7] = 1
    assert flags() == 0
    h[11] = float("nan")
    tokens[11] = 5
    assert flags() == B.MLS_DEVFLAG_NONFINITE and torch.isnan(logp[11])


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 2048), (torch.float32, 128)])
def test_vocabulary_chunks(dtype, d):
    """One chunk, and chunks that the vocabulary does not fill: the same gradients."""
    h, W, tokens, gl = _draw(200, d, 3000, dtype, 5)
    for chunk in (256, 1024, 1 << 20):
        _check(h, W, tokens, gl, 0.9, _run(h, W, tokens, gl, temperature=0.9, vocab_chunk=chunk), f"chunk {chunk}")


def test_wide_logits():
    """Logits from -200 to 200: log-probabilities far below what exp represents."""
    h, W, tokens, gl = _draw(64, 64, 1000, torch.float32, 6, ignore=0.0)
    W = W * 30
    logp, entropy, gh, gW = _run(h, W, tokens, gl)
    lp, en = P.token_logp(_np(h), _np(W), tokens.cpu().numpy())
    assert lp.min() < -100
    np.testing.assert_allclose(_np(logp), lp, rtol=1e-6, atol=1e-4)
    np.testing.assert_allclose(_np(entropy), en, atol=1e-4)
    assert torch.isfinite(gh).all() and torch.isfinite(gW).all()


def test_one_gradient_alone_and_no_gradient():
    h, W, tokens, gl = _draw(150, 64, 900, torch.bfloat16, 7)
    logp, entropy, gh, gW = _run(h, W, tokens, gl)
    h1 = h.detach().requires_grad_(True)
    assert torch.equal(torch.autograd.grad(D.token_logp(h1, W, tokens)[0], h1, gl)[0], gh)
    W1 = W.detach().requires_grad_(True)
    assert torch.equal(torch.autograd.grad(D.token_logp(h, W1, tokens)[0], W1, gl)[0], gW)
    with torch.no_grad():
        lp, en = D.token_logp(h1, W1, tokens)
    assert not lp.requires_grad and torch.equal(lp, logp) and torch.equal(en, entropy)


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                       (torch.bfloat16, torch.float32)])
def test_accumulated_gradients(dtype, out):
    """grad_h and grad_W += : the sum's own rounding once, ignored tokens' rows as they were."""
    h, W, tokens, gl = _draw(300, 64, 900, dtype, 11)
    flags = B.MLS_GRAD_W_BF16 if out == torch.bfloat16 else 0
    g0 = [torch.randn(x.shape, device=DEV).to(out) for x in (h, W)]

    def grads(acc):
        p = D.make_problem([h], [W], tokens, grad_h_dtype=out, flags=flags | acc)
        stats = torch.empty(B.query_sizes(p)[1], dtype=torch.uint8, device=DEV)
        logp, s = torch.empty(300, device=DEV), D._stream(h.device)
        ws = torch.full((max(B.token_logp_workspace(p)[:2]),), 255, dtype=torch.uint8, device=DEV)
        B.token_logp_fwd(p, stats.data_ptr(), logp.data_ptr(), None, None, ws.data_ptr(), ws.numel(), s)
        g = [x.clone() if acc else torch.full_like(x, float("nan")) for x in g0]
        ws.fill_(255)
        B.token_logp_bwd(p, stats.data_ptr(), None, gl.data_ptr(), g[0].data_ptr(), g[1].data_ptr(), ws.data_ptr(),
                         ws.numel(), s)
        torch.cuda.synchronize()
        return g
    plain, acc = grads(0), grads(B.MLS_ACCUMULATE_GRAD_H | B.MLS_ACCUMULATE_GRAD_W)
    half = 2.0 ** -8 if out == torch.bfloat16 else 2.0 ** -24
    # sizes that a sum may pass through on its way: the magnitudes of its terms
    G = torch.softmax(h.double() @ W.double().t(), 1)
    live = tokens != -100
    G[live, tokens[live]] = 1 - G[live, tokens[live]]
    G *= (gl.double().abs() * live)[:, None]
    sizes = G @ W.double().abs(), G.t() @ h.double().abs()
    for a, b, c, size in zip(plain, g0, acc, sizes):
        a, b, c = a.double(), b.double(), c.double()
        # the plain gradient's rounding and the sum's; an fp32 grad_W starts its sum over 300 tokens at the old
        # value, so each of its 19 products of 16 tokens rounds at the size of that value and of the terms so far,
        # which their sum of magnitudes bounds (the end of the sum may be far smaller), twice at most: 2^-24 * 40
        n = 40 if out == torch.float32 else 4
        s = size if out == torch.float32 else a.abs() + c.abs()
        assert bool(((c - (a + b)).abs() <= n * half * (s + b.abs())).all())
    ignored = tokens == -100
    assert torch.equal(acc[0][ignored], g0[0][ignored]) and not plain[0][ignored].any()


def test_a_head_used_twice_collects_both_gradients():
    h, W, tokens, gl = _draw(150, 64, 900, torch.float32, 8)
    h2 = torch.roll(h, 3, 0)
    W1 = W.detach().requires_grad_(True)
    a, b = D.token_logp(h, W1, tokens)[0], D.token_logp(h2, W1, tokens)[0]
    (a @ gl + b @ gl).backward()
    ref = P.token_logp_backward(_np(h), _np(W), tokens.cpu().numpy(), _np(gl))[1] + \
        P.token_logp_backward(_np(h2), _np(W), tokens.cpu().numpy(), _np(gl))[1]
    assert_grad_rows(_np(W1.grad), ref, "shared head")


def test_hidden_states_of_4_gib():
    """Packed rows that reach 4 GiB take the general gradient kernels (64-bit addresses)."""
    T, d, V = 131200, 16384, 260
    g = torch.Generator(device=DEV).manual_seed(12)
    h = torch.empty(T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    W = (torch.randn(V, d, generator=g, device=DEV) * 0.01).bfloat16()
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV)
    tokens[::3] = -100
    h[::3] = float("nan")
    gl = torch.randn(T, generator=g, device=DEV)
    logp, entropy, gh, gW = _run(h, W, tokens, gl, temperature=0.8)
    Wd, rW = W.double(), torch.zeros(V, d, dtype=torch.float64, device=DEV)
    for t0 in range(0, T, 16384):
        rows = t0 + (tokens[t0:t0 + 16384] != -100).nonzero()[:, 0]
        hd, y = h[rows].double(), tokens[rows]
        lp = torch.log_softmax(hd @ Wd.t() / 0.8, 1)
        assert (logp[rows] - lp.gather(1, y[:, None])[:, 0]).abs().max() <= 1e-4
        G = -lp.exp()
        G[torch.arange(rows.numel(), device=DEV), y] += 1
        G *= (gl[rows].double() / 0.8)[:, None]
        rh = G @ Wd
        assert (gh[rows].double() - rh).norm() <= 2e-2 * rh.norm()
        rW += G.t() @ hd
    assert not gh[::3].any() and not logp[::3].any()
    assert (gW.double() - rW).norm() <= 2e-2 * rW.norm()


def test_gradient_against_differences():
    """Along random directions, in float32: (f(h + e v) - f(h - e v)) / 2e is v . grad.
    A difference of sums of about 40 fp32 log-probabilities of size 8 is off by at most
    40 * 8 * 2^-20 / 2e, the third derivative costs e^2."""
    h, W, tokens, gl = _draw(40, 64, 300, torch.float32, 9)
    _, _, gh, gW = _run(h, W, tokens, gl, temperature=0.8)
    g = torch.Generator(device=DEV).manual_seed(1)
    f = lambda a, b: float((D.token_logp(a, b, tokens, temperature=0.8)[0].double() * gl.double()).sum())  # noqa: E731
    for x, grad, at in ((h, gh, lambda v: f(v, W)), (W, gW, lambda v: f(h, v))):
        v = torch.randn(x.shape, generator=g, device=DEV)
        v /= v.norm()
        e = 0.05
        num = (at(x + e * v) - at(x - e * v)) / (2 * e)
        assert abs(num - float((grad.double() * v.double()).sum())) <= 40 * 8 * 2.0 ** -20 / (2 * e) + 10 * e * e


def test_refusals():
    h, W, tokens, _ = _draw(10, 64, 50, torch.bfloat16, 10)
    for bad in (dict(h=h.float()), dict(h=h[:, :32]), dict(h=h.t()), dict(W=W[:, ::2]), dict(tokens=tokens.int()),
                dict(tokens=tokens[:5]), dict(h=h[0])):
        with pytest.raises((ValueError, RuntimeError)):
            D.token_logp(**{"h": h, "W": W, "tokens": tokens, **bad})
    for t in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(B.MlsError):
            D.token_logp(h, W, tokens, temperature=t)
