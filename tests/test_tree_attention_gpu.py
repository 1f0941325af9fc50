"""Attention of a tree of drafted tokens over a paged cache, against the float64 oracle."""

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2608_09703_amd import api as D
from tests.tree_helpers import DEV, Cache, tree, values

pytestmark = pytest.mark.gpu


def _fill(rng, c, dtype, parents, odd=None):
    """Entries of the context and of the tree's nodes; returns the oracle's lists. Nodes that are not there
    keep the pool's NaN."""
    k, v = [], []
    for b in range(c.B):
        kb, vb = [], []
        L = int(c.lengths[b])
        for t in range(max(L, 0) + c.n if L >= 0 else 0):
            x, y = values(rng, (c.heads, c.D), dtype), values(rng, (c.heads, c.D), dtype)
            if t >= L:
                if parents is not None and O.way_up(parents[b], t - L) is None:
                    kb.append(None)
                    vb.append(None)
                    continue
                if odd is not None:
                    y = odd(b, t - L, y)
            c.put(b, t, x, y)
            kb.append(x)
            vb.append(y)
        k.append(kb)
        v.append(vb)
    return k, v


def _bound(q, k, v, lengths, parents, dtype, want):
    """Rounding errors: with W = sum w |v| / sum w and S the largest sum |q k| scale,
    bf16: each weight up to 2^-8 off, the result rounded by up to 2^-8 of itself;
    both: fp32 scores (D + 4 roundings of up to S, twice: numerator and sum), fp32 sums of as many terms as entries."""
    Dh = q.shape[3]
    absk = [[None if x is None else np.abs(x) for x in b] for b in k]
    absv = [[None if x is None else np.abs(x) for x in b] for b in v]
    W = O.attention(q, k, absv, lengths, parents)
    S = 1.0
    for b in range(len(absk)):
        for x in absk[b]:
            if x is not None:
                g = q.shape[2] // x.shape[0]
                S = max(S, float((np.abs(q[b]).reshape(q.shape[1], -1, g, Dh) * x[:, None, :]).sum(-1).max()) * Dh ** -0.5)
    n = max(len(b) for b in k) + 8
    f32 = 2 * (Dh + 4) * 2.0 ** -24 * S * 1.5 + n * 2.0 ** -24
    if dtype == torch.bfloat16:
        return 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + f32) * W * (1 + 2.0 ** -7)
    return f32 * W + 2.0 ** -23 * np.abs(want)


def _check(got, want, bound):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf])
    rest = np.isfinite(want)
    err = np.abs(got[rest] - want[rest])
    assert (err <= bound[rest] + 1e-30).all(), float((err - bound[rest]).max())


CASES = [
    # dtype, D, kv heads, group, n, page, lengths, layout
    ("bf16", 64, 2, 1, 1, 16, [0, 1, 15, 16, 17], "heads_first"),
    ("bf16", 128, 2, 1, 7, 16, [0, 33, 250, 255], "heads_first"),
    ("bf16", 96, 3, 1, 16, 16, [5, 300, -1, 31], "entries_first"),
    ("bf16", 32, 1, 2, 9, 32, [40, 0], "padded"),
    ("bf16", 192, 1, 3, 5, 64, [70, 3], "heads_first"),
    ("bf16", 256, 1, 1, 40, 16, [100], "heads_first"),
    ("bf16", 256, 1, 4, 3, 16, [20, 50], "heads_first"),
    ("bf16", 128, 1, 2, 64, 128, [129, 200], "heads_first"),
    ("bf16", 64, 1, 8, 13, 16, [77], "heads_first"),  # more rows than a tile
    ("bf16", 96, 1, 1, 3, 16, [1500, 2, 700], "heads_first"),  # several parts
    # more rows of a key head than a tile
    ("bf16", 128, 1, 8, 9, 16, [0, 40, 127], "heads_first"),
    ("bf16", 96, 1, 4, 40, 16, [900, 15], "padded"),
    ("f32", 64, 3, 4, 9, 32, [0, 1, 90, 333], "heads_first"),
    ("f32", 32, 1, 1, 33, 16, [47, 48], "entries_first"),
    ("f32", 96, 2, 1, 20, 16, [130], "heads_first"),
    ("f32", 128, 1, 5, 4, 16, [64, 9], "padded"),
    ("f32", 128, 1, 1, 50, 16, [30], "heads_first"),
    ("f32", 192, 1, 1, 2, 16, [700, 5], "heads_first"),
    ("f32", 192, 1, 1, 20, 16, [40], "heads_first"),
    ("f32", 256, 1, 1, 18, 16, [260], "heads_first"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_against_the_oracle(case):
    dt, Dh, hk, group, n, page, lengths, layout = case
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    rng = np.random.default_rng(sum(lengths) + 1000 * n + Dh)
    c = Cache(rng, lengths, n, hk, Dh, page, dtype, layout=layout)
    parents = tree(rng, c.B, n)
    k, v = _fill(rng, c, dtype, parents)
    q = values(rng, (c.B, n, hk * group, Dh), dtype, 2.0)
    got = D.tree_attention(torch.tensor(q, device=DEV).to(dtype), *c.layer(), torch.tensor(parents, device=DEV))
    want = O.attention(q, k, v, lengths, parents)
    _check(got, want, _bound(q, k, v, lengths, parents, dtype, want))


WIDE = [
    # tiles of 64 rows, of 32 and of 16
    ("bf16", 32, 1, 1, 64, 16, [20, 300], "heads_first"), ("bf16", 64, 1, 2, 25, 16, [33, 290], "padded"),
    ("bf16", 64, 2, 1, 20, 32, [7], "heads_first"), ("bf16", 96, 2, 1, 30, 16, [0, 520], "heads_first"),
    ("bf16", 128, 1, 2, 16, 64, [15, 260, -1], "entries_first"), ("bf16", 192, 1, 1, 40, 16, [18, 280], "heads_first"),
    ("bf16", 256, 1, 1, 20, 16, [270], "heads_first"), ("f32", 32, 1, 1, 50, 16, [16, 300], "heads_first"),
    ("f32", 64, 1, 3, 11, 16, [31, 270], "heads_first"), ("f32", 96, 1, 1, 40, 16, [261], "heads_first"),
    ("f32", 128, 1, 1, 20, 32, [9, 256], "padded"), ("f32", 192, 1, 1, 33, 16, [258], "heads_first"),
    ("f32", 256, 1, 1, 18, 16, [12, 257], "heads_first"), ("bf16", 128, 3, 1, 5, 16, [300, 1], "heads_first"),
    # more than 64 rows of a key head: a block's waves share the entries
    ("bf16", 128, 1, 8, 9, 16, [0, 40, 127, 128], "heads_first"), ("bf16", 64, 2, 5, 33, 64, [63, 700, -1], "entries_first"),
    ("bf16", 96, 1, 4, 40, 16, [900, 15], "padded"), ("bf16", 128, 1, 3, 64, 32, [64, 300], "heads_first"),
    ("bf16", 64, 1, 8, 64, 16, [31, 255], "heads_first"), ("bf16", 96, 3, 5, 14, 16, [33], "heads_first"),
    ("f32", 64, 1, 8, 17, 16, [40, 258], "heads_first"), ("bf16", 192, 1, 5, 20, 16, [50], "heads_first")]


@pytest.mark.parametrize("room", [512 * 256, 1 << 21])
@pytest.mark.parametrize("case", WIDE, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_wide_tables(case, room):
    """Tables with room for many parts: the largest tiles of rows, and (the wider one) loads past the caches."""
    dt, Dh, hk, group, n, page, lengths, layout = case
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    rng = np.random.default_rng(sum(lengths) + 1000 * n + Dh)
    c = Cache(rng, lengths, n, hk, Dh, page, dtype, layout=layout)
    parents = tree(rng, c.B, n)
    k, v = _fill(rng, c, dtype, parents)
    table = torch.full((c.B, room // page), -1, dtype=torch.int32, device=DEV)
    table[:, :c.per] = c.t_table
    q = values(rng, (c.B, n, hk * group, Dh), dtype, 2.0)
    got = D.tree_attention(torch.tensor(q, device=DEV).to(dtype), c.k[0], c.v[0], table, c.t_lengths,
                           torch.tensor(parents, device=DEV))
    want = O.attention(q, k, v, lengths, parents)
    _check(got, want, _bound(q, k, v, lengths, parents, dtype, want))


@pytest.mark.parametrize("Dh", [32, 64, 128])
def test_many_calls_give_the_same_bits(Dh):
    """Sequences whose nodes lie in a wave's third tile: every call is right, and equal to the first."""
    rng = np.random.default_rng(64332 + Dh)
    n, lengths = 64, [20, 300]
    c = Cache(rng, lengths, n, 1, Dh, 16, torch.bfloat16)
    parents = tree(rng, c.B, n)
    k, v = _fill(rng, c, torch.bfloat16, parents)
    table = torch.full((c.B, (1 << 20) // 16), -1, dtype=torch.int32, device=DEV)
    table[:, :c.per] = c.t_table
    q = values(rng, (c.B, n, 1, Dh), torch.bfloat16, 2.0)
    args = (torch.tensor(q, device=DEV).to(torch.bfloat16), c.k[0], c.v[0], table, c.t_lengths,
            torch.tensor(parents, device=DEV))
    got = [D.tree_attention(*args) for _ in range(300)]
    want = O.attention(q, k, v, lengths, parents)
    _check(got[0], want, _bound(q, k, v, lengths, parents, torch.bfloat16, want))
    for x in got[1:]:
        assert torch.equal(x.view(torch.int16), got[0].view(torch.int16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_chain_strides_and_scale(dtype):
    """Without parents a node sees the earlier ones; q lies in a wider tensor; a scale of the caller's."""
    rng = np.random.default_rng(3)
    c = Cache(rng, [21, 50], 6, 2, 64, 16, dtype)
    chain = np.tile(np.arange(-1, 5, dtype=np.int32), (2, 1))
    k, v = _fill(rng, c, dtype, chain)
    q = values(rng, (2, 6, 4, 64), dtype)
    qkv = torch.full((2, 6, 3, 4, 64), float("nan"), dtype=dtype, device=DEV)
    qkv[:, :, 1] = torch.tensor(q, device=DEV).to(dtype)
    got = D.tree_attention(qkv[:, :, 1], *c.layer(), scale=0.03)
    want = O.attention(q, k, v, [21, 50], chain, scale=0.03)
    _check(got, want, _bound(q, k, v, [21, 50], chain, dtype, want))
    assert torch.equal(got, D.tree_attention(qkv[:, :, 1], *c.layer(), torch.tensor(chain, device=DEV), scale=0.03))


@pytest.mark.parametrize("dtype,heads", [(torch.bfloat16, 2), (torch.float32, 2), (torch.bfloat16, 9)])
@pytest.mark.parametrize("length", [3, 300])  # in one part, and in several
def test_infinities_reach_the_rows_that_see_them_only(dtype, heads, length):
    rng = np.random.default_rng(9)
    n = 8
    c = Cache(rng, [length], n, 1, 64, 16, dtype, wide=20)
    parents = np.array([[-1, 0, 0, 1, 1, 2, -1, 6]], np.int32)
    marks = {1: (3, np.inf), 2: (3, -np.inf), 4: (60, np.nan), 3: (3, -np.inf), 6: (0, np.inf)}

    def odd(b, i, y):
        if i in marks:
            y = y.copy()
            y[:, marks[i][0]] = marks[i][1]
        return y
    k, v = _fill(rng, c, dtype, parents, odd)
    q = values(rng, (1, n, heads, 64), dtype)
    table = c.t_table
    if heads > 8:  # (room for many parts: a block's waves share the entries)
        table = torch.full((1, 5000), -1, dtype=torch.int32, device=DEV)
        table[:, :c.per] = c.t_table
    got = D.tree_attention(torch.tensor(q, device=DEV).to(dtype), c.k[0], c.v[0], table, c.t_lengths,
                           torch.tensor(parents, device=DEV))
    want = O.attention(q, k, v, [length], parents)
    assert np.isinf(want).any() and np.isnan(want).any() and np.isfinite(want).any()
    plain = [[np.where(np.isfinite(x), x, 0.0) for x in b] for b in v]
    _check(got, want, _bound(q, k, plain, [length], parents, dtype, np.where(np.isfinite(want), want, 0.0)))


def test_keys_that_are_not_finite():
    """A node's own NaN or infinite key makes its rows NaN; siblings do not see it."""
    rng = np.random.default_rng(10)
    c = Cache(rng, [40], 4, 1, 64, 16, torch.bfloat16)
    parents = np.array([[-1, -1, -1, 2]], np.int32)
    k, v = _fill(rng, c, torch.bfloat16, parents)
    q = values(rng, (1, 4, 1, 64), torch.bfloat16)
    c.put(0, 41, np.full((1, 64), np.nan), v[0][41])
    got = D.tree_attention(torch.tensor(q, device=DEV).to(torch.bfloat16), *c.layer(), torch.tensor(parents, device=DEV))
    want = O.attention(q, k, v, [40], parents)
    want[0, 1] = np.nan
    _check(got, want, _bound(q, k, v, [40], parents, torch.bfloat16, np.nan_to_num(want)))


def test_scores_of_very_different_sizes():
    """Maxima that grow along the entries by far more than a weight's range, and equal scores."""
    rng = np.random.default_rng(11)
    n, L = 2, 600
    c = Cache(rng, [L], n, 1, 64, 16, torch.float32)
    parents = np.array([[-1, 0]], np.int32)
    q = np.zeros((1, n, 1, 64))
    q[..., 0] = 8.0
    k, v = [[]], [[]]
    for t in range(L + n):
        x = np.zeros((1, 64))
        x[0, 0] = float(t // 100) * 200.0  # scores 0, 200, 400 ...: only the last run counts
        y = values(rng, (1, 64), torch.float32)
        c.put(0, t, x, y)
        k[0].append(x)
        v[0].append(y)
    got = D.tree_attention(torch.tensor(q, device=DEV).float(), *c.layer(), torch.tensor(parents, device=DEV))
    want = O.attention(q, k, v, [L], parents)
    np.testing.assert_allclose(got.cpu().numpy(), want, rtol=0, atol=3 * 2.0 ** -23 * 4)


def test_scores_near_the_lowest_number():
    """Rows whose scores are all next to float32's lowest number still weigh them against one another."""
    rng = np.random.default_rng(3)
    c = Cache(rng, [20], 1, 1, 32, 16, torch.float32)
    k, v = np.zeros((21, 1, 32)), values(rng, (21, 1, 32), torch.float32)
    k[:, 0, 0] = np.float32(-2.3e19)
    k[[4, 17], 0, 0] = np.float32(-2.2e19)
    for t in range(21):
        c.put(0, t, k[t], v[t])
    q = torch.zeros(1, 1, 1, 32, device=DEV)
    q[..., 0] = 1e19
    got = D.tree_attention(q, *c.layer(), scale=1.0)[0, 0, 0].double().cpu().numpy()
    # (in base 2 the scores are -3.32e38 and -3.17e38: all weight is on the two; two sums and a quotient in fp32)
    want = (v[4, 0] + v[17, 0]) / 2
    assert np.abs(got - want).max() <= 3 * 2.0 ** -24 * np.abs(v).max()


def test_pages_that_are_not_there():
    rng = np.random.default_rng(12)
    n = 3
    c = Cache(rng, [70, 40, 60, 50], n, 1, 32, 16, torch.float32)
    parents = np.tile(np.array([-1, 0, 1], np.int32), (4, 1))
    k, v = _fill(rng, c, torch.float32, parents)
    table = c.table.copy()
    table[0, 1] = -1               # entries 16 .. 31
    table[1, 0] = c.pages          # entries 0 .. 15
    table[2, :] = 2 ** 31 - 1      # none
    for t in range(16, 32):
        k[0][t] = None
    for t in range(16):
        k[1][t] = None
    k[2] = [None] * len(k[2])
    q = values(rng, (4, n, 2, 32), torch.float32)
    got = D.tree_attention(torch.tensor(q, device=DEV).float(), c.k[0], c.v[0], torch.tensor(table, device=DEV),
                           c.t_lengths, torch.tensor(parents, device=DEV))
    want = O.attention(q, k, v, [70, 40, 60, 50], parents)
    _check(got, want, _bound(q, k, v, [70, 40, 60, 50], parents, torch.float32, want))
    assert (got[2] == 0).all()


@pytest.mark.parametrize("pages", [2, 40])  # in one part, and in several
@pytest.mark.parametrize("past", [0, 1, 500, 2 ** 31 - 1])
def test_lengths_past_the_table(pages, past):
    """A context that fills the table's row or goes beyond it: what the row names is the context, the nodes are not
    there."""
    rng = np.random.default_rng(pages)
    n, room = 5, 16 * pages
    c = Cache(rng, [room - n], n, 1, 32, 16, torch.float32)
    assert c.per == pages
    chain = np.array([np.arange(-1, n - 1)], np.int32)
    k, v = _fill(rng, c, torch.float32, chain)
    lengths = torch.tensor([min(room + past, 2 ** 31 - 1)], dtype=torch.int32, device=DEV)
    q = values(rng, (1, n, 2, 32), torch.float32)
    got = D.tree_attention(torch.tensor(q, device=DEV).float(), c.k[0], c.v[0], c.t_table, lengths)
    k, v = ([x[0] + [None] * n] for x in (k, v))
    want = O.attention(q, k, v, [room], chain)
    _check(got, want, _bound(q, k, v, [room], chain, torch.float32, want))


def test_streams_graphs_and_repeats():
    """The same bits on every call, on another stream, and from a captured graph with other inputs in place."""
    rng = np.random.default_rng(13)
    c = Cache(rng, [900, 33], 12, 2, 64, 16, torch.bfloat16)
    parents = torch.tensor(tree(rng, 2, 12), device=DEV)
    _fill(rng, c, torch.bfloat16, parents.cpu().numpy())
    q = torch.tensor(values(rng, (2, 12, 2, 64), torch.bfloat16), device=DEV).bfloat16()
    want = D.tree_attention(q, *c.layer(), parents)
    for _ in range(3):
        assert torch.equal(D.tree_attention(q, *c.layer(), parents), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = D.tree_attention(q, *c.layer(), parents)
    side.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = D.tree_attention(q, *c.layer(), parents)
    for i in range(3):
        q.mul_(0.5 if i else 1.0)
        c.t_lengths[0] = 900 - 300 * i
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, D.tree_attention(q, *c.layer(), parents))


@pytest.mark.parametrize("group,Dh,room", [(3, 128, 512 * 256), (1, 96, 1 << 21), (5, 64, 1 << 19)])
def test_wide_tables_in_a_graph_and_on_two_streams(group, Dh, room):
    """Replays follow new lengths, trees and queries; two calls at once do not share a workspace."""
    rng = np.random.default_rng(group)
    n, page, lengths = 40, 16, [290, 44]
    c = Cache(rng, [310, 60], n, 1, Dh, page, torch.bfloat16)  # (room for the longer contexts below)
    parents = tree(rng, c.B, n, absent=False)
    _fill(rng, c, torch.bfloat16, parents)
    table = torch.full((c.B, room // page), -1, dtype=torch.int32, device=DEV)
    table[:, :c.per] = c.t_table
    make = lambda: torch.tensor(values(rng, (c.B, n, group, Dh), torch.bfloat16), device=DEV).to(torch.bfloat16)  # noqa: E731
    q, len_, par = make(), torch.tensor(lengths, dtype=torch.int32, device=DEV), torch.tensor(parents, device=DEV)
    call = lambda x, ln, pr: D.tree_attention(x, c.k[0], c.v[0], table, ln, pr)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(q, len_, par)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call(q, len_, par)
    for step in range(3):
        q.copy_(make())
        len_.copy_(torch.tensor([[290, 44], [310, 60], [-1, 7]][step], dtype=torch.int32))
        par.copy_(torch.tensor(tree(rng, c.B, n), device=DEV))
        g.replay()
        assert torch.equal(out.view(torch.int16), call(q, len_, par).view(torch.int16))
    other = make()
    want = call(q, len_, par).clone(), call(other, len_, par).clone()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(side):
            b = call(other, len_, par)
        a = call(q, len_, par)
        torch.cuda.synchronize()
        assert torch.equal(a.view(torch.int16), want[0].view(torch.int16))
        assert torch.equal(b.view(torch.int16), want[1].view(torch.int16))
