"""Several children of a node on rows of all sizes: a register's token to a thread, lists of more than 1,024 tokens
(top_p = 1, or a flat rest within the nucleus), rows opened beforehand and by the walk. Uniforms lie just below and
just above each child's threshold."""

import numpy as np
import pytest
import torch

from oracle import decode as C
from oracle import tree as O
from paper_2608_09703_amd import api as D

DEV = "cuda:0"
pytestmark = pytest.mark.gpu

HEAD = np.array([0.4, 0.2, 0.12, 0.08, 0.05, 0.03])  # of the children's tokens, the rest is flat
# the draft's: what is left of p stays between 0 and q at the first four children, each in its turn
DRAFT = np.array([0.4715, 0.194, 0.1063, 0.066, 0.074, 0.0348])
TURN_DOWN = 1.0 - 2.0 ** -24
# a threshold in 64 bits against the kernel's: weights 2e-14 off and sums of up to 65,536 of them 65,536 x 2^-53;
# the float32 uniform beside it is placed 2^-20 of it away, rounded by 2^-24 of it
NEAR = 2.0 ** -20


def _rows(rng, V, at, head=HEAD):
    """float32 logits with the probabilities `head` at the tokens `at` and a rest that differs by up to 20 %."""
    p = np.full(V, 1.0) + 0.2 * rng.random(V)
    p[at] = 0.0
    p *= (1.0 - head.sum()) / p.sum()
    p[at] = head
    return (np.log(p) + 3.0).astype(np.float32)


def _thresholds(p, q, children):
    """What u is held against for each child after those before it were turned down, from the formula itself."""
    out = []
    for x in children:
        out.append(p[x] / (q[x] if q is not None else 1.0))
        left = np.maximum(p - q, 0.0) if q is not None else np.where(np.arange(p.size) == x, 0.0, p)
        p = left / left.sum()
    return out


# V, top_p, trees (0: two to a child, their rows opened beforehand; else so many, opened by the walk)
CASES = [(64, 1.0, 0), (64, 0.98, 0), (1500, 1.0, 0), (1500, 0.999, 0), (49152, 1.0, 0), (4096, 0.97, 0), (65536, 1.0, 0),
         (64, 1.0, 600), (1500, 1.0, 600), (1500, 0.999, 600)]


@pytest.mark.parametrize("sampled", [False, True])
@pytest.mark.parametrize("V,top_p,trees", CASES)
def test_uniforms_on_either_side_of_each_threshold(V, top_p, trees, sampled):
    rng = np.random.default_rng(V + trees + sampled)
    m = len(HEAD)
    at = rng.permutation(V)[:m]
    row = _rows(rng, V, at)
    top = float(np.float32(top_p))
    p = C.filtered_probs(row, 1.0, top)
    drow, q = None, None
    if sampled:
        drow = _rows(rng, V, at, DRAFT)
        q = C.filtered_probs(drow, 1.0, top)
    marks = _thresholds(p, q, at)
    B, n = trees or 2 * m, m + 1
    parents = np.tile(np.array([-1] + [0] * m, np.int32), (B, 1))
    tokens = np.tile(np.concatenate([[0], at]).astype(np.int32), (B, 1))
    ua = np.full((B, n), TURN_DOWN, np.float32)
    child = np.arange(B) // 2 % m
    below = np.arange(B) % 2 == 0
    reach = np.full(B, -1)  # the child that has to be taken
    for b in range(B):
        j = int(child[b])
        u = marks[j] * (1.0 - NEAR if below[b] else 1.0 + NEAR)
        ua[b, 1 + j] = min(u, TURN_DOWN)
        for i in range(m):
            if float(ua[b, 1 + i]) < marks[i]:
                reach[b] = i
                break
        else:
            reach[b] = m
    us = rng.random(B).astype(np.float32)
    target = torch.tensor(row, device=DEV).expand(B, n, V).contiguous()
    draft = torch.tensor(drow, device=DEV).expand(B, n, V).contiguous() if sampled else None
    got = D.tree_verify(target, torch.tensor(tokens, device=DEV), torch.tensor(parents, device=DEV),
                        torch.tensor(ua, device=DEV), torch.tensor(us, device=DEV), draft_logits=draft, temperature=1.0,
                        top_p=top_p)
    acc, path, nxt = (x.cpu().numpy() for x in got)
    np.testing.assert_array_equal(acc, (reach < m).astype(int))
    np.testing.assert_array_equal(path[:, 1], np.where(reach < m, reach + 1, -1))
    few = np.arange(B) if B <= 2 * m else np.arange(0, B, 37)
    want = O.verify(np.broadcast_to(row, (len(few), n, V)), tokens[few], parents[few], ua[few], us[few], 1.0, top,
                    np.broadcast_to(drow, (len(few), n, V)) if sampled else None)
    for g, w in zip((acc, path, nxt), want):
        np.testing.assert_array_equal(g[few], w)
    assert set(reach) == set(range(4 if sampled else m)) | {m}  # every child's threshold is met from both sides


@pytest.mark.parametrize("V,top_p", [(64, 1.0), (1100, 1.0), (1500, 0.999)])
def test_first_tokens_follow_the_verifiers_distribution(V, top_p):
    """30,000 walks with the most likely tokens proposed. A frequency is off by its deviation, sqrt(p (1 - p) / N) <=
    0.0029; 5 of them are passed once in a million and a half times."""
    rng = np.random.default_rng(V)
    N, m = 30000, 4
    at = rng.permutation(V)[:len(HEAD)]
    row = _rows(rng, V, at)
    p = C.filtered_probs(row, 1.0, float(np.float32(top_p)))
    n = m + 1
    target = torch.tensor(row, device=DEV).expand(N, n, V).contiguous()
    tokens = torch.tensor(np.concatenate([[0], at[:m]]).astype(np.int32), device=DEV).expand(N, n).contiguous()
    parents = torch.tensor([-1] + [0] * m, dtype=torch.int32, device=DEV).expand(N, n).contiguous()
    acc, path, nxt = D.tree_verify(target, tokens, parents, torch.tensor(rng.random((N, n)), dtype=torch.float32, device=DEV),
                                   torch.tensor(rng.random(N), dtype=torch.float32, device=DEV), top_p=top_p)
    first = torch.where(acc > 0, tokens.gather(1, path[:, 1:2].clamp(min=0).long())[:, 0], nxt).cpu().numpy()
    got = np.bincount(first, minlength=V) / N
    for x in at:
        assert abs(got[x] - p[x]) < 5.0 * np.sqrt(p[x] * (1.0 - p[x]) / N), (x, got[x], p[x])
    rest = 1.0 - p[at].sum()
    assert abs(1.0 - got[at].sum() - rest) < 5.0 * np.sqrt(rest * (1.0 - rest) / N)
