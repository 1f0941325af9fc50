"""Verification of drafted trees, against the float64 oracle: whole numbers, which have to be equal."""

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2608_09703_amd import api as D
from paper_2608_09703_amd import binding as B
from tests.tree_helpers import DEV, tree

pytestmark = pytest.mark.gpu


def _inputs(rng, Bt, n, V, temperature, sampled, close=0.4):
    parents = tree(rng, Bt, n)
    parents[:, 0] = -1
    target = (rng.standard_normal((Bt, n, V)) * 2).astype(np.float32)
    draft = (target + close * rng.standard_normal((Bt, n, V))).astype(np.float32)
    tokens = rng.integers(0, V, (Bt, n)).astype(np.int32)
    for b in range(Bt):
        for i in range(1, n):
            p = parents[b, i]
            row = draft[b, p if 0 <= p < i else 0].astype(np.float64) / temperature
            if sampled:
                tokens[b, i] = int(np.argmax(row + rng.gumbel(size=V)))
            else:
                tokens[b, i] = int(np.argsort(-row)[int((parents[b, :i] == p).sum()) % V])
    return (parents, target, draft, tokens, rng.random((Bt, n)).astype(np.float32), rng.random(Bt).astype(np.float32))


def _gpu(*xs):
    return [torch.tensor(x, device=DEV) if x is not None else None for x in xs]


def _run(parents, target, draft, tokens, ua, us, **kw):
    out = D.tree_verify(*_gpu(target, tokens, parents, ua, us), draft_logits=_gpu(draft)[0], **kw)
    return [x.cpu().numpy() for x in out]


def _same(got, want):
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g, w)


@pytest.mark.parametrize("Bt,n,V,temperature,top_p,sampled", [
    (5, 1, 700, 0.4, 0.9, True), (6, 9, 1000, 0.4, 0.9, True), (4, 33, 2111, 1.0, 0.95, True),
    (3, 64, 1024, 0.7, 1.0, True), (4, 20, 1500, 1.0, 1.0, False), (6, 9, 1000, 0.7, 0.9, False),
    (2, 7, 49152, 0.4, 0.9, True), (1, 5, 65536, 1.0, 1.0, True), (3, 6, 2, 1.0, 1.0, True)])
def test_against_the_oracle(Bt, n, V, temperature, top_p, sampled):
    rng = np.random.default_rng(V + n)
    taken = 0
    for _ in range(3):
        parents, target, draft, tokens, ua, us = _inputs(rng, Bt, n, V, temperature, sampled)
        got = _run(parents, target, draft if sampled else None, tokens, ua, us, temperature=temperature, top_p=top_p)
        want = O.verify(target, tokens, parents, ua, us, float(np.float32(temperature)), float(np.float32(top_p)),
                        draft if sampled else None)
        _same(got, want)
        taken += int(want[0].sum())
    assert n == 1 or V == 2 or taken > 0


@pytest.mark.parametrize("Bt,n,V", [(5, 12, 1000), (2, 64, 300), (3, 4, 50304)])
def test_greedy(Bt, n, V):
    rng = np.random.default_rng(n)
    taken = 0
    for i in range(8):
        parents, target, draft, tokens, ua, us = _inputs(rng, Bt, n, V, 1.0, False, close=0.05)
        if i % 2 == 0:
            target[:, :, V // 2] = target.max(2)  # ties: the lowest index
        want = O.verify(target, tokens, parents, ua, us, 1.0, 1.0, greedy=True)
        _same(_run(parents, target, None, tokens, None, None, greedy=True), want)
        taken += int(want[0].sum())
    assert taken > 0


@pytest.mark.parametrize("V,top_p,sampled", [(300, 0.9, True), (1500, 1.0, True), (1500, 1.0, False)])
def test_more_trees_than_rows_are_opened_beforehand(V, top_p, sampled):
    rng = np.random.default_rng(V)
    Bt, n = 530, 4
    parents, target, draft, tokens, ua, us = _inputs(rng, Bt, n, V, 0.7, sampled)
    got = _run(parents, target, draft if sampled else None, tokens, ua, us, temperature=0.7, top_p=top_p)
    _same(got, O.verify(target, tokens, parents, ua, us, float(np.float32(0.7)), float(np.float32(top_p)),
                        draft if sampled else None))


def test_a_chain_gives_what_chain_verification_gives():
    rng = np.random.default_rng(5)
    Bt, G, V = 40, 5, 1200
    parents = np.tile(np.arange(-1, G, dtype=np.int32), (Bt, 1))
    _, target, draft, tokens, ua, us = _inputs(rng, Bt, G + 1, V, 0.7, True)
    for b in range(Bt):
        for i in range(1, G + 1):
            tokens[b, i] = int(np.argmax(draft[b, i - 1] / 0.7 + rng.gumbel(size=V)))
    t, dr, tok, u = _gpu(target, draft, tokens, ua)
    n1, x1 = D.spec_verify(dr[:, :G].transpose(0, 1).contiguous(), t, tok[:, 1:].t().contiguous(),
                           u[:, 1:].t().contiguous(), torch.tensor(us, device=DEV), temperature=0.7, top_p=0.95)
    for par in (parents, None):
        n2, path, x2 = _run(par, target, draft, tokens, ua, us, temperature=0.7, top_p=0.95)
        np.testing.assert_array_equal(n2, n1.cpu().numpy())
        np.testing.assert_array_equal(x2, x1.cpu().numpy())
        np.testing.assert_array_equal(path, np.where(np.arange(G + 1) <= n2[:, None], np.arange(G + 1), -1))


def test_records_of_the_sampler_and_tokens_out_of_range():
    rng = np.random.default_rng(6)
    Bt, n, V = 4, 10, 900
    parents, target, draft, tokens, ua, us = _inputs(rng, Bt, n, V, 0.7, True)
    tokens[0, 1:4] = [-1, V, 2 ** 31 - 1]
    kw = dict(temperature=0.7, top_p=0.9)
    got = _run(parents, target, draft, tokens, ua, us, **kw)
    _same(got, O.verify(target, tokens, parents, ua, us, float(np.float32(0.7)), float(np.float32(0.9)), draft))
    rec = torch.empty(Bt * n * B.ROW_PARAMS_BYTES, dtype=torch.uint8, device=DEV)
    D.sample(torch.tensor(draft, device=DEV).view(Bt * n, V), torch.zeros(Bt * n, device=DEV), params=rec, **kw)
    _same(_run(parents, target, draft, tokens, ua, us, draft_params=rec, **kw), got)
    _same(_run(parents, target, None, tokens, ua, us, **kw),
          O.verify(target, tokens, parents, ua, us, float(np.float32(0.7)), float(np.float32(0.9))))


def test_equal_distributions_and_repeated_children():
    """p = q takes every child that it can produce; a token offered twice without probabilities cannot be taken
    the second time; mass that runs out leaves p as it was."""
    rng = np.random.default_rng(7)
    Bt, n, V = 6, 8, 64
    parents, target, draft, tokens, ua, us = _inputs(rng, Bt, n, V, 1.0, True, close=0.0)
    parents[:] = 0
    parents[:, 0] = -1
    kw = dict(temperature=1.0, top_p=1.0)
    got = _run(parents, target, target, tokens, ua, us, **kw)
    assert (got[0] == 1).all() and (got[1][:, 1] == 1).all()
    tokens[:] = tokens[:, :1]
    ua[:, 1] = 1.0 - 2.0 ** -24
    ua[:, 2:] = 0.0
    _same(_run(parents, target, None, tokens, ua, us, **kw), O.verify(target, tokens, parents, ua, us, 1.0, 1.0))
    target[:, 0] = -np.inf  # all mass on one token, which is offered, turned down (u q = p), and drawn
    target[:, 0, 5] = 0.0
    tokens[:] = 5
    tokens[:, 1] = 6
    got = _run(parents, target, target, tokens, np.ones_like(ua), us, **kw)
    assert (got[2] >= 0).all()
    _same(got, O.verify(target, tokens, parents, np.ones_like(ua), us, 1.0, 1.0, target))


def test_rows_without_a_distribution():
    rng = np.random.default_rng(8)
    Bt, n, V = 4, 5, 300
    parents, target, draft, tokens, ua, us = _inputs(rng, Bt, n, V, 1.0, True)
    target[0] = np.nan
    target[1] = -np.inf
    target[2, :, 7] = np.inf
    for d in (draft, None):
        got = _run(parents, target, d, tokens, ua, us, temperature=0.5, top_p=0.9)
        assert (got[0][:3] == 0).all() and (got[2][:3] == -1).all() and got[2][3] >= 0
    got = _run(parents, target, None, tokens, None, None, greedy=True)
    assert (got[2][:2] == -1).all() and got[2][2] == 7 and (got[0][:2] == 0).all()


def test_streams_and_graphs():
    rng = np.random.default_rng(9)
    parents, target, draft, tokens, ua, us = _inputs(rng, 8, 12, 3000, 0.7, True)
    t, tok, par, a, s, dr = _gpu(target, tokens, parents, ua, us, draft)
    kw = dict(draft_logits=dr, temperature=0.7, top_p=0.9)
    want = D.tree_verify(t, tok, par, a, s, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = D.tree_verify(t, tok, par, a, s, **kw)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = D.tree_verify(t, tok, par, a, s, **kw)
    for i in range(3):
        s.copy_(torch.rand(8, device=DEV))
        a.copy_(torch.rand(8, 12, device=DEV))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, D.tree_verify(t, tok, par, a, s, **kw)))
