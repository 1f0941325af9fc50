"""Inputs of the tests of decoding with a tree of drafted tokens."""

import numpy as np
import torch

DEV = "cuda:0"


def tree(rng, B, n, absent=True):
    """Random parents: mostly earlier nodes, some behind the context, and (absent) some that are no node's."""
    p = np.zeros((B, n), np.int32)
    for b in range(B):
        for i in range(n):
            p[b, i] = rng.integers(-1, i) if i else -1
            if absent and rng.random() < 0.15:
                p[b, i] = rng.choice([-2, i, i + 1, 100, -2 ** 31])
    return p


class Cache:
    """A pool full of NaN, and sequences of the given lengths in pages in no order."""

    def __init__(self, rng, lengths, n, heads, D, page, dtype, layers=1, layout="heads_first", spare=3, wide=0):
        self.B, self.n, self.heads, self.D, self.page, self.layers = len(lengths), n, heads, D, page, layers
        need = max(max(lengths), 0) + n
        self.per = -(-need // page) + wide
        self.pages = self.B * self.per + spare
        self.table = rng.permutation(self.pages)[:self.B * self.per].reshape(self.B, self.per).astype(np.int32)
        self.lengths = np.array(lengths, np.int32)
        shape = (layers, self.pages, heads, page, D)
        if layout == "entries_first":  # [.., page, heads, D] as a view with the heads in front
            make = lambda: torch.full((layers, self.pages, page, heads, D), float("nan"), dtype=dtype,  # noqa: E731
                                      device=DEV).transpose(2, 3)
        elif layout == "padded":  # columns of a wider tensor
            make = lambda: torch.full((layers, self.pages, heads, page, 2 * D), float("nan"), dtype=dtype,  # noqa: E731
                                      device=DEV)[..., D // 2:D // 2 + D]
        else:
            make = lambda: torch.full(shape, float("nan"), dtype=dtype, device=DEV)  # noqa: E731
        self.k, self.v = make(), make()
        self.t_table = torch.tensor(self.table, device=DEV)
        self.t_lengths = torch.tensor(self.lengths, device=DEV)

    def at(self, b, t):
        return int(self.table[b, t // self.page]), t % self.page

    def put(self, b, t, k, v, layer=0):
        """k, v: [heads, D] float64 values that the dtype holds."""
        pg, e = self.at(b, t)
        self.k[layer, pg, :, e] = torch.tensor(k, device=DEV).to(self.k.dtype)
        self.v[layer, pg, :, e] = torch.tensor(v, device=DEV).to(self.v.dtype)

    def layer(self, i=0):
        return self.k[i], self.v[i], self.t_table, self.t_lengths


def values(rng, shape, dtype, scale=1.0):
    """float64 values that the dtype holds."""
    x = torch.tensor(rng.standard_normal(shape) * scale, dtype=torch.float32).to(dtype)
    return x.double().numpy()
