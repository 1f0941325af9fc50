"""The operators together, as a server uses them: decoding steps with drafted trees give the tokens and the cache of
decoding one token at a time."""

import pytest
import torch

from paper_2608_09703_amd import api as D
from tests.tree_helpers import DEV

pytestmark = pytest.mark.gpu

V, H, HK, HD, PAGE = 211, 4, 2, 32, 16
STEPS = 24


class Model:
    """One attention layer over embeddings: keys, values and queries are tables over the tokens."""

    def __init__(self, dtype):
        g = torch.Generator(device=DEV)
        g.manual_seed(5)
        rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        self.dtype = dtype
        self.q = (rnd(V, H, HD) * 2).to(dtype)
        self.k, self.v = rnd(V, HK, HD).to(dtype), rnd(V, HK, HD).to(dtype)
        self.W, self.s = D.quantize_rows(rnd(V, H * HD).to(dtype))

    def logits(self, tokens, kp, vp, table, lengths, parents=None):
        """Writes the nodes' entries, attends and returns [B, n, V]."""
        B, n = tokens.shape
        D.cache_write(self.k[tokens], self.v[tokens], kp, vp, table, lengths)
        o = D.tree_attention(self.q[tokens], kp, vp, table, lengths, parents)
        return D.head_logits_int8(o.view(B * n, H * HD), self.W, self.s).view(B, n, V)


def _pool(B, entries):
    per = -(-entries // PAGE)
    g = torch.Generator().manual_seed(7)
    table = torch.randperm(B * per + 2, generator=g)[:B * per].view(B, per).to(torch.int32).to(DEV)
    return table, B * per + 2


def _decode(m, first, table, pages):
    """One token at a time: the tokens [B, STEPS + 1] and the pages."""
    B = first.numel()
    kp = torch.zeros(pages, HK, PAGE, HD, dtype=m.dtype, device=DEV)
    vp = torch.zeros_like(kp)
    out = [first]
    for t in range(STEPS):
        lengths = torch.full((B,), t, dtype=torch.int32, device=DEV)
        logits = m.logits(out[-1][:, None], kp, vp, table, lengths)
        out.append(D.sample(logits.view(B, V), None, greedy=True).long())
    return torch.stack(out, 1), kp, vp


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_trees_give_the_tokens_of_plain_decoding(dtype):
    B, n = 5, 9
    m = Model(dtype)
    first = torch.arange(B, device=DEV) * 17 % V
    table, pages = _pool(B, STEPS + 1 + n)
    want, kp1, vp1 = _decode(m, first, table, pages)
    kp = torch.zeros(1, pages, HK, PAGE, HD, dtype=dtype, device=DEV)
    vp = torch.zeros_like(kp)
    lengths = torch.zeros(B, dtype=torch.int32, device=DEV)
    got = [[int(x)] for x in first]
    g = torch.Generator().manual_seed(3)
    accepted = 0
    for _ in range(STEPS):
        # two children per node; one of them is the right token now and then
        parents = torch.tensor([[-1, 0, 0, 1, 1, 2, 2, 3, 3]] * B, dtype=torch.int32)
        tokens = torch.randint(0, V, (B, n), generator=g)
        for b in range(B):
            at = {0: len(got[b]) - 1}
            tokens[b, 0] = got[b][-1]
            for i in range(1, n):
                at[i] = at[int(parents[b, i])] + 1
                if torch.rand(1, generator=g) < 0.6 and at[i] <= STEPS:
                    tokens[b, i] = want[b, at[i]]
        parents[4, 5:] = -2  # a smaller tree
        tok, par = tokens.to(DEV), parents.to(DEV)
        logits = m.logits(tok, kp[0], vp[0], table, lengths, par)
        n_acc, path, nxt = D.tree_verify(logits, tok.to(torch.int32), par, None, None, greedy=True)
        lengths = D.cache_compact(kp, vp, table, lengths, path, n_acc)
        for b in range(B):
            if int(lengths[b]) < 0:
                continue
            got[b] += [int(tokens[b, int(path[b, j])]) for j in range(1, int(n_acc[b]) + 1)] + [int(nxt[b])]
            accepted += int(n_acc[b])
            assert int(lengths[b]) == len(got[b]) - 1
            if len(got[b]) > STEPS:
                lengths[b] = -1  # done: takes no part
    assert accepted > B * 4
    for b in range(B):
        assert got[b][:STEPS + 1] == want[b].tolist()
    for b in range(B):
        for t in range(STEPS):
            pg, e = int(table[b, t // PAGE]), t % PAGE
            assert torch.equal(kp[0, pg, :, e], kp1[pg, :, e]) and torch.equal(vp[0, pg, :, e], vp1[pg, :, e])


def test_a_step_in_one_graph():
    """Write, attend, head, verify and compact captured once and replayed as the lengths grow."""
    B, n = 3, 5
    m = Model(torch.bfloat16)
    table, pages = _pool(B, 200)
    parents = torch.tensor([[-1, 0, 0, 1, 3]] * B, dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    tokens = torch.randint(0, V, (B, n), generator=g, device=DEV)
    u, us = torch.rand(B, n, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)

    def step(kp, vp, lengths):
        logits = m.logits(tokens, kp[0], vp[0], table, lengths, parents)
        n_acc, path, nxt = D.tree_verify(logits, tokens.to(torch.int32), parents, u, us, temperature=0.7, top_p=0.9)
        return n_acc, path, nxt, D.cache_compact(kp, vp, table, lengths, path, n_acc)

    pools = [torch.zeros(1, pages, HK, PAGE, HD, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    lengths = torch.zeros(B, dtype=torch.int32, device=DEV)
    eager_lengths = lengths.clone()
    step(pools[2].clone(), pools[3].clone(), lengths.clone())  # (every kernel is loaded)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(pools[0], pools[1], lengths)
    for i in range(4):
        tokens.copy_(torch.randint(0, V, (B, n), generator=g, device=DEV))
        u.copy_(torch.rand(B, n, generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        want = step(pools[2], pools[3], eager_lengths)
        assert all(torch.equal(x, y) for x, y in zip(out, want))
        assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
        lengths.copy_(out[3])
        eager_lengths = want[3]
