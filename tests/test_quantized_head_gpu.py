"""Rows as 8-bit integers and the head product on them, against the float64 oracle."""

import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2608_09703_amd import api as D
from tests.tree_helpers import DEV

pytestmark = pytest.mark.gpu


def _rows(T, d, dtype, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + T + d)
    return (torch.randn(T, d, generator=g, device=DEV) * torch.exp(torch.randn(T, 1, generator=g, device=DEV))).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(1, 1), (3, 7), (5, 16), (70, 1001), (9, 4352), (2, 20000), (300, 64)])
def test_quantize(T, d, dtype):
    x = _rows(T, d, dtype)
    q, s = D.quantize_rows(x)
    wq, ws = O.quantize(x.double().cpu().numpy())
    np.testing.assert_array_equal(s.double().cpu().numpy(), ws)
    np.testing.assert_array_equal(q.cpu().numpy(), wq)


def test_quantize_edges():
    """Zeros, ties (to even), the smallest numbers, rows that lie apart, infinities and NaN."""
    x = torch.zeros(9, 24, device=DEV)
    x[1, :8] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -126.5], device=DEV)
    x[2, :3] = torch.tensor([1e-45, -3e-45, 190 * 1.4e-45], device=DEV)
    x[3, :2] = torch.tensor([3.4e38, -1e38], device=DEV)
    x[4, 5] = float("nan")
    x[5, 6] = float("inf")
    x[6, 7] = -float("inf")
    x[7] = -1.0
    x[8, 0] = 1e-45
    wide = torch.full((9, 50), float("nan"), device=DEV)
    wide[:, 3:27] = x
    want_q, want_s = O.quantize(np.where(np.isfinite(x.double().cpu().numpy()), x.double().cpu().numpy(), 0.0))
    for rows in (x, wide[:, 3:27]):
        q, s = D.quantize_rows(rows)
        assert torch.isnan(s[4:7]).all() and (q[4:7] == 0).all()
        keep = [0, 1, 2, 3, 7, 8]
        np.testing.assert_array_equal(s.double().cpu().numpy()[keep], want_s[keep])
        np.testing.assert_array_equal(q.cpu().numpy()[keep], want_q[keep])


# every tile: up to 32, 64 and more rows, few and many vocabulary rows, four token tiles, widths past a K-tile
@pytest.mark.parametrize("T,d,V", [(1, 16, 5), (1, 4352, 3000), (32, 256, 1001), (33, 1008, 700), (64, 128, 4099),
                                   (65, 272, 2000), (102, 1024, 33000), (129, 144, 33001), (500, 384, 9000),
                                   (700, 112, 12001)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_head(T, d, V, dtype):
    o = _rows(T, d, dtype)
    W, s = D.quantize_rows(_rows(V, d, dtype, 5) * 0.05)
    got = D.head_logits_int8(o, W, s)
    q, so = O.quantize(o.double().cpu().numpy())
    want = (torch.tensor(q, device=DEV) @ W.double().t()) * torch.tensor(so, device=DEV)[:, None] * s.double()
    # the sum's conversion and two products: three roundings of up to 2^-24
    assert ((got.double() - want).abs() <= 3.01 * 2.0 ** -24 * want.abs()).all()


def test_head_rows_that_are_not_finite():
    o = _rows(40, 64, torch.bfloat16)
    W, s = D.quantize_rows(_rows(300, 64, torch.bfloat16, 1))
    want = D.head_logits_int8(o, W, s)
    o[3, 9], o[17, 0] = float("nan"), float("inf")
    got = D.head_logits_int8(o, W, s)
    rest = [t for t in range(40) if t not in (3, 17)]
    assert torch.isnan(got[3]).all() and torch.isnan(got[17]).all() and torch.equal(got[rest], want[rest])


def test_extreme_sums():
    """All products of one sign: the largest sum of the widest rows stays in 32 bits."""
    d = 1 << 17
    o = torch.ones(2, d, device=DEV)
    o[1] = -1.0
    W = torch.full((9, d), 127, dtype=torch.int8, device=DEV)
    got = D.head_logits_int8(o, W, torch.ones(9, device=DEV))
    want = 127.0 * 127.0 * d * float(np.float32(1 / 127.0))
    assert torch.allclose(got[0].double(), torch.full((9,), want, dtype=torch.float64, device=DEV), rtol=2.0 ** -22)
    assert torch.equal(got[1], -got[0])


def test_out_streams_and_graphs():
    o = _rows(6, 256, torch.bfloat16)
    W, s = D.quantize_rows(_rows(2000, 256, torch.bfloat16, 1))
    want = D.head_logits_int8(o, W, s)
    out = torch.empty(6, 2000, device=DEV)
    assert D.head_logits_int8(o, W, s, out) is out and torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = D.head_logits_int8(o, W, s)
    side.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = D.head_logits_int8(o, W, s)
    for i in range(3):
        o.mul_(-1.0 - i)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, D.head_logits_int8(o, W, s))
