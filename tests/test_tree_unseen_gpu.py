"""What a node does not see does not change a bit of its result: another node's key that moves that node's maximum, by
little and past 2^20, that is infinite or NaN, or values that are."""

import numpy as np
import pytest
import torch

from paper_2608_09703_amd import api as D
from tests.tree_helpers import DEV, Cache, values

pytestmark = pytest.mark.gpu

CASES = [
    # dtype, D, kv heads, group, n, lengths, table's room in entries (0: the lengths')
    ("bf16", 64, 2, 1, 9, [700, 33], 0), ("bf16", 128, 1, 2, 16, [300, 1200], 1 << 21), ("bf16", 32, 1, 1, 64, [130], 1 << 17),
    ("bf16", 128, 1, 8, 16, [257, 40], 1 << 21), ("bf16", 96, 1, 4, 40, [500], 1 << 21), ("bf16", 256, 1, 1, 12, [90, 0], 0),
    ("f32", 64, 2, 2, 11, [333, 5], 0), ("f32", 128, 1, 1, 20, [700], 1 << 17), ("f32", 192, 1, 1, 7, [64, 800], 0)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_another_nodes_entry(case):
    dt, Dh, hk, group, n, lengths, room = case
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    rng = np.random.default_rng(Dh + n + sum(lengths))
    page = 16
    c = Cache(rng, lengths, n, hk, Dh, page, dtype)
    for b in range(c.B):
        for t in range(lengths[b] + n):
            c.put(b, t, values(rng, (hk, Dh), dtype), values(rng, (hk, Dh), dtype))
    table = c.t_table
    if room:
        table = torch.full((c.B, room // page), -1, dtype=torch.int32, device=DEV)
        table[:, :c.per] = c.t_table
    # a chain, and in the middle of it a node that nothing else sees
    odd = n // 2
    parents = np.tile(np.arange(-1, n - 1, dtype=np.int32), (c.B, 1))
    parents[:, odd + 1] = odd - 1
    parents = torch.tensor(parents, device=DEV)
    q = torch.tensor(values(rng, (c.B, n, hk * group, Dh), dtype, 2.0), device=DEV).to(dtype)
    run = lambda: D.tree_attention(q, c.k[0], c.v[0], table, c.t_lengths, parents)  # noqa: E731
    want = run()
    others = [i for i in range(n) if i != odd]
    assert torch.isfinite(want).all()
    ks, vs = c.k.clone(), c.v.clone()
    own = q[0, odd].view(hk, group, Dh)[:, 0].double().cpu().numpy()
    changed = 0
    for key, value in ((0.02 * own, None), (own, None), (8.0 * own, None), (1e6 * own, None), (1e30 * own, None),
                       (-1e30 * own, None), (np.inf * np.ones_like(own), None), (np.nan * own, None),
                       (own, np.inf * np.ones_like(own)), (own, np.nan * own)):
        c.k.copy_(ks)
        c.v.copy_(vs)
        for b in range(c.B):
            pg, e = c.at(b, lengths[b] + odd)
            c.k[0, pg, :, e] = torch.tensor(key, device=DEV).to(dtype)
            if value is not None:
                c.v[0, pg, :, e] = torch.tensor(value, device=DEV).to(dtype)
        got = run()
        changed += not torch.equal(got[:, odd], want[:, odd])
        bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
        assert torch.equal(got[:, others].view(bits), want[:, others].view(bits))
    assert changed >= 8
