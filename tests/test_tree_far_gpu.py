"""Decoding with a tree of drafted tokens: arrays whose offsets do not fit 32 bits."""

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2608_09703_amd import api as D
from tests.tree_helpers import DEV, tree, values

pytestmark = pytest.mark.gpu
FAR = 1 << 31


def test_cache_and_attention():
    """Pages more than 2^31 elements from the first one, in either layout of heads and entries."""
    rng = np.random.default_rng(0)
    B, n, heads, Dh, page = 2, 5, 2, 64, 16
    lengths = [37, 300]
    for step in (FAR // 600 // 64 * 64, page * heads * Dh):  # few pages far apart; many pages
        pages = FAR // step + 40
        k_pool = torch.empty(pages * step, dtype=torch.bfloat16, device=DEV)
        v_pool = torch.empty(pages * step, dtype=torch.bfloat16, device=DEV)
        view = lambda x: x.as_strided((pages, heads, page, Dh), (step, page * Dh, Dh, 1))  # noqa: E731
        kp, vp = view(k_pool), view(v_pool)
        per = 20
        table = torch.tensor(pages - 1 - rng.permutation(B * per).reshape(B, per), dtype=torch.int32, device=DEV)
        assert int(table.min()) * step > FAR // 2 and int(table.max()) * step > FAR
        total = max(lengths) + n
        k, v = (values(rng, (B, total, heads, Dh), torch.bfloat16) for _ in range(2))
        t_len = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        t_k, t_v = (torch.tensor(x, device=DEV).to(torch.bfloat16) for x in (k, v))
        # the contexts, then the nodes behind them
        D.cache_write(t_k, t_v, kp, vp, table, torch.zeros_like(t_len), counts=t_len)
        new = [torch.stack([x[b, lengths[b]:lengths[b] + n] for b in range(B)]) for x in (t_k, t_v)]
        D.cache_write(*new, kp, vp, table, t_len)
        parents = tree(rng, B, n, absent=False)
        q = values(rng, (B, n, 4, Dh), torch.bfloat16)
        got = D.tree_attention(torch.tensor(q, device=DEV).to(torch.bfloat16), kp, vp, table, t_len,
                               torch.tensor(parents, device=DEV))
        want = O.attention(q, k, v, lengths, parents)
        # weights and the result in bf16, half a step each; fp32 sums of 305 terms
        bound = (2.0 ** -8 + 2.0 ** -8) * np.abs(v).max() + 1e-3
        assert np.abs(got.double().cpu().numpy() - want).max() <= bound
        path = torch.tensor([[0, 2, 4, -1, -1], [0, 3, -1, -1, -1]], dtype=torch.int32, device=DEV)
        length = D.cache_compact(kp, vp, table, t_len, path, torch.tensor([2, 1], dtype=torch.int32, device=DEV))
        assert length.tolist() == [40, 302]
        for b, j, node in ((0, 1, 2), (0, 2, 4), (1, 1, 3)):
            t = lengths[b] + j
            for pool, x in ((kp, t_k), (vp, t_v)):
                assert torch.equal(pool[table[b, t // page].long(), :, t % page], x[b, lengths[b] + node])
        del kp, vp, k_pool, v_pool


@pytest.mark.parametrize("B,n,V", [(900, 64, 40000), (500, 64, 65536)])  # no, and one row of a tree opened beforehand
def test_verification(B, n, V):
    rng = np.random.default_rng(1)
    target = torch.empty(B, n, V, dtype=torch.float32, device=DEV)
    assert target.numel() * 4 > 3 * FAR
    rows = rng.standard_normal((2, V)).astype(np.float32) * 3
    target[:, 0] = torch.tensor(rows[0], device=DEV)
    target[B - 1, 0] = torch.tensor(rows[1], device=DEV)
    tokens = torch.arange(n, dtype=torch.int32, device=DEV).repeat(B, 1)
    ua = torch.ones(B, n, device=DEV)  # nothing is taken
    us = torch.full((B,), 0.37, device=DEV)
    parents = torch.full((B, n), -2, dtype=torch.int32, device=DEV)
    parents[:, 1:3] = 0
    acc, path, nxt = D.tree_verify(target, tokens, parents, ua, us, temperature=0.7, top_p=0.9)
    assert int(acc.abs().sum()) == 0 and torch.equal(path[:, 1:], torch.full_like(path[:, 1:], -1))
    want = [int(O.verify(rows[r].reshape(1, 1, V).repeat(3, 1), np.arange(3)[None], np.array([[-1, 0, 0]]),
                         np.ones((1, 3), np.float32), np.array([0.37], np.float32), float(np.float32(0.7)),
                         float(np.float32(0.9)))[2][0]) for r in range(2)]
    assert nxt[:B - 1].tolist() == [want[0]] * (B - 1) and int(nxt[B - 1]) == want[1]


def test_rows_and_head():
    d = 1 << 16
    T = FAR // d + 3
    x = torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    x.normal_()
    q, s = D.quantize_rows(x)
    assert q.numel() > FAR
    for t in (0, T - 2, T - 1):
        wq, ws = O.quantize(x[t:t + 1].double().cpu().numpy())
        np.testing.assert_array_equal(q[t].cpu().numpy(), np.asarray(wq)[0])
        assert float(s[t]) == float(np.asarray(ws)[0])
    del x, q, s
    V, d = 131072, 16
    T = FAR // V + 5
    W, ws = D.quantize_rows(torch.randn(V, d, device=DEV))
    o = torch.randn(T, d, device=DEV)
    logits = D.head_logits_int8(o, W, ws)
    assert logits.numel() > FAR
    oq, os_ = D.quantize_rows(o)
    for t in (0, T - 1):
        want = (oq[t].double() @ W.double().T) * os_[t].double() * ws.double()
        # two factors rounded to fp32 on the way
        assert float(((logits[t].double() - want).abs() - 3 * 2.0 ** -24 * want.abs()).max()) <= 1e-30
